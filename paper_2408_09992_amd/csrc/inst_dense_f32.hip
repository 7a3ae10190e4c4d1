// Instantiates the dense cross entropy's kernels for one type of W and queries.
#define PQ_DENSE_INSTANCE float
#include "default_cross_entropy.hpp"
