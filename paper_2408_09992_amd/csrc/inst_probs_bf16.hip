// Instantiates the dense log-probabilities' kernels for one type of W and queries.
#define PQ_PROBS_INSTANCE __bf16
#include "default_log_probs.hpp"
