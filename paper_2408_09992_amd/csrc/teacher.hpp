// A teacher's list of one position as probabilities, by one wave, and its items' scores by W phi, in 64 bits (512 entries at most: nothing beside a pass over the items).
#pragma once
#include "head_common.hpp"

namespace pqk {
namespace head {

constexpr int kMostEntries = 512;

// A number of every thread, joined over the workgroup by `f` (which does not ask for an order); `part` is shared, a place a wave.
template <int THREADS, typename V, typename F>
__device__ __forceinline__ V over_workgroup(V v, V* part, F f) {
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) v = f(v, __shfl_xor(v, x));
    __syncthreads();
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / kWave; ++w) v = f(v, part[w]);
    return v;
}

// A list by one wave, which keeps no entry: the largest score over T, the sum of the exponentials and its logarithm.
struct WaveTeacher {
    double top, sum, log_sum;
    bool any;
    // of an entry's score over T less `top`
    __device__ __forceinline__ double weight(double x) const { return x == -__builtin_inf() ? 0.0 : exp(x) / sum; }
};
// x(k): the k-th entry's score over T, -inf where there is no entry.
template <typename X>
__device__ __forceinline__ WaveTeacher wave_teacher(int K, X x_of) {
    WaveTeacher t{-__builtin_inf(), 0.0, 0.0, false};
    for (int k = (int)threadIdx.x % kWave; k < K; k += kWave) {
        const double x = x_of(k);
        t.any |= x != -__builtin_inf();
        t.top = fmax(t.top, x);
    }
    t.any = __any(t.any);
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) t.top = fmax(t.top, __shfl_xor(t.top, x));
    if (!t.any) return t;
    for (int k = (int)threadIdx.x % kWave; k < K; k += kWave) {
        const double x = x_of(k);
        if (x != -__builtin_inf()) t.sum += exp(x - t.top);
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) t.sum += __shfl_xor(t.sum, x);
    t.log_sum = log(t.sum);
    return t;
}
__device__ __forceinline__ WaveTeacher wave_teacher(const int* items, const float* scores, int q, int K, long long N, float temperature) {
    return wave_teacher(K, [&](int k) {
        const int item = items[(size_t)q * K + k];
        return item >= 0 && item < N ? (double)scores[(size_t)q * K + k] / (double)temperature : -__builtin_inf();
    });
}

// What an entry adds to sum_k w_k (log w_k - log p_k), log p_k = score / T - lse.
__device__ __forceinline__ double entry_loss(double weight, double log_weight, double score, float temperature, double lse) {
    return weight == 0.0 ? 0.0 : weight * (log_weight - (counted(score / (double)temperature) - lse));
}

// Rows of W by one query in 64 bits (products of 16-bit elements are exact, and nearly always their sum): sums of d products by sixteen lanes of a wave, which
// all sixteen get, of two rows at once, whose loads are on their way together.  Rows are multiples of 16 bytes, and aligned.
template <typename T>
__device__ __forceinline__ void dots64(const T* x0, const T* x1, const T* y, int d, double& sum0, double& sum1) {
    constexpr int kOf = 16 / (int)sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(kOf)));
    sum0 = sum1 = 0.0;
    constexpr int kAtOnce = 4;                                  // pieces of each row that a lane has on their way
    const int pieces = d / kOf;
    for (int first = (int)threadIdx.x % 16; first < pieces; first += 16 * kAtOnce) {
        Piece u0[kAtOnce], u1[kAtOnce], v[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int i = min(first + 16 * j, pieces - 1);
            u0[j] = reinterpret_cast<const Piece*>(x0)[i];
            u1[j] = reinterpret_cast<const Piece*>(x1)[i];
            v[j] = reinterpret_cast<const Piece*>(y)[i];
        }
        __builtin_amdgcn_sched_barrier(0);                     // (not one piece after the other)
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (first + 16 * j >= pieces) break;
#pragma unroll
            for (int e = 0; e < kOf; ++e) {
                sum0 = fma((double)(float)u0[j][e], (double)(float)v[j][e], sum0);
                sum1 = fma((double)(float)u1[j][e], (double)(float)v[j][e], sum1);
            }
        }
    }
#pragma unroll
    for (int w = 1; w < 16; w *= 2) {
        sum0 += __shfl_xor(sum0, w);
        sum1 += __shfl_xor(sum1, w);
    }
}
// The same of the rows item(0 .. n - 1) (below 0: none), by the threads FROM .. TO - 1 of a workgroup; put(i, whether there is one, sum) by one lane each.
template <int FROM, int TO, typename T, typename Item, typename Put>
__device__ __forceinline__ void score_rows(const T* W, const T* h, int d, int n, Item item, Put put) {
    constexpr int kRows = (TO - FROM) / 16;
    for (int i = ((int)threadIdx.x - FROM) / 16; i < n; i += 2 * kRows) {
        const bool two = i + kRows < n;
        const long long r0 = item(i), r1 = two ? item(i + kRows) : -1;       // (the same for the sixteen)
        double s0, s1;
        if (r0 >= 0 || r1 >= 0) dots64(W + (size_t)(r0 >= 0 ? r0 : r1) * d, W + (size_t)(r1 >= 0 ? r1 : r0) * d, h, d, s0, s1);
        if (threadIdx.x % 16 == 0) {
            put(i, r0 >= 0, s0);
            if (two) put(i + kRows, r1 >= 0, s1);
        }
    }
}

}  // namespace head
}  // namespace pqk
