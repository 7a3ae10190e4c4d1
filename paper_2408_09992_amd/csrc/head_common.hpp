// What the kernels that train the scoring head share: constants, cross-lane steps, the host's checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pqk {

// pqtopk.hip: keeps HIP's text for pq_strerror() and returns PQ_ERR_HIP, or PQ_OK for hipSuccess.
__attribute__((visibility("hidden"))) int record_hip_error(hipError_t e);

namespace head {

constexpr int kWave = 64;
constexpr int kCUs = 256;                            // MI355X; only sizes grids and workspaces
constexpr size_t kMaxLds = 160 * 1024;               // LDS per workgroup on gfx950
constexpr double kLog2eDouble = 1.4426950408889634;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32: 1 ulp, results below 2^-126 become 0

// Keeps a branch that is rarely taken a branch: the compiler otherwise runs both sides and selects.
__device__ __forceinline__ void stay_a_branch() { asm volatile("; rare" ::: "memory"); }

// Orders a wave's LDS accesses (LDS serves a wave's requests in the order in which they were made).
__device__ __forceinline__ void wave_reads_after_writes() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A sum of exponentials held as reference and mantissa: total = s * 2^c.  The reference is kept within +-2^23, where float32 resolves
// a half: 2^(x log2e - c) is the exact product's distance from it, so with a rounded reference far outside (a mask of -1e30) the terms
// would be 2 to the power of that rounding, inf or 0.  Scores below the range so count as -inf, those above it as +inf.
constexpr float kLowest = -8388608.0f, kHighest = 8388608.0f;
// A score over T whose exponential is 0 over any reference (2^-126 and what lies below it are): as a log-probability, too, it is -inf.
constexpr double kLeastScore = ((double)kLowest - 126.0) / kLog2eDouble;
__device__ __forceinline__ double counted(double x) { return x < kLeastScore ? -__builtin_inf() : x; }      // (a NaN stays one)
// Of a score over T: at most 0, also where the sums' rounding has the likeliest item over that.
__device__ __forceinline__ float log_prob_of(double x, double lse) {
    const double v = counted(x) - lse;
    return lse == -__builtin_inf() ? -__builtin_inff() : v > 0.0 ? 0.0f : (float)v;
}
__device__ __forceinline__ void join_sums(float& c, float& s, float c2, float s2) {
    const float top = fmaxf(c, c2);
    s = s * exp2_fast(c - top) + s2 * exp2_fast(c2 - top);
    c = top;
}
// The reference moves up to `top`, the largest of the next scores (base 2; +inf too), where these pass it by more than there is room for.
__device__ __forceinline__ void raise_reference(float& c, float& s, float top) {
    const float to = fminf(top, kHighest);
    s *= exp2_fast(c - to);
    c = to;
}
// Besides, a sum of terms 2^x x (what an entropy is made of): total = 2^c (t + c s).  A term's x is held over -200, where 2^x is 0 and -inf would make NaN.
// An entropy is the small difference of log2 s and t / s where few items have most of the mass, so the reference stays near the largest score.
constexpr float kNearHeadroom = 4.0f;
__device__ __forceinline__ float weighted(float p, float x, float t) { return fmaf(p, fmaxf(x, -200.0f), t); }
__device__ __forceinline__ void join_sums(float& c, float& s, float& t, float c2, float s2, float t2) {
    const float top = fmaxf(c, c2), f = exp2_fast(c - top), f2 = exp2_fast(c2 - top);
    t = f * fmaf(c - top, s, t) + f2 * fmaf(c2 - top, s2, t2);
    s = s * f + s2 * f2;
    c = top;
}
__device__ __forceinline__ void raise_reference(float& c, float& s, float& t, float top) {
    const float to = fminf(top, kHighest), f = exp2_fast(c - to);
    t = f * fmaf(c - to, s, t);
    s *= f;
    c = to;
}
// Those of OF lanes of a wave, which all of them get.
template <int OF = kWave>
__device__ __forceinline__ void join_wave(float& c, float& s, float& t) {
#pragma unroll
    for (int x = 1; x < OF; x *= 2) join_sums(c, s, t, __shfl_xor(c, x), __shfl_xor(s, x), __shfl_xor(t, x));
}
// - sum_i p log p in nats: log p = ln 2 (x - log2 s).  0 where no score counts.
__device__ __forceinline__ float entropy_of(float s, float t) {
    return s == 0.0f ? 0.0f : s < __builtin_inff() ? (float)fmax((log2((double)s) - (double)t / (double)s) / kLog2eDouble, 0.0) : __builtin_nanf("");
}
// log-sum: -inf where no score counts, NaN where one is NaN, +inf or counts as that.
__device__ __forceinline__ float log_sum(float c, float s) {
    return s == 0.0f ? -__builtin_inff() : s < __builtin_inff() ? (c + __log2f(s)) * kLn2 : __builtin_nanf("");
}

// The same in 64 bits: reference and logarithm of some 20 each lose no bits to their sum.  to_nats: 1 over what scores were multiplied with, times T.  That factor is
// log2 e / T rounded to 24 bits, so by ln 2 itself the log-sum would be off by up to 2^-24 of itself, and a score over T less it by as much.
__device__ __forceinline__ double log_sum64(float c, float s, double to_nats) {
    return s == 0.0f ? -__builtin_inf() : s < __builtin_inff() ? ((double)c + log2((double)s)) * to_nats : __builtin_nan("");
}
inline double base_of(float scale, float temperature) { return (double)scale * (double)temperature; }

template <typename F>
inline hipError_t allow_lds(F* kernel, size_t bytes) {
    if (bytes <= 64 * 1024) return hipSuccess;
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

// Temperatures and how many items a position may be given (pqtopk_probs.h).
constexpr int kMostGiven = 65536;
inline bool temperature_fits(float t) { return t >= 1e-4f && t <= 1e4f; }

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }
inline size_t round_up(size_t a, size_t to) { return (a + to - 1) / to * to; }

}  // namespace head
}  // namespace pqk
