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
// log-sum: -inf where no score counts, NaN where one is NaN, +inf or counts as that.
__device__ __forceinline__ float log_sum(float c, float s) {
    return s == 0.0f ? -__builtin_inff() : s < __builtin_inff() ? (c + __log2f(s)) * kLn2 : __builtin_nanf("");
}

template <typename F>
inline hipError_t allow_lds(F* kernel, size_t bytes) {
    if (bytes <= 64 * 1024) return hipSuccess;
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }
inline size_t round_up(size_t a, size_t to) { return (a + to - 1) / to * to; }

}  // namespace head
}  // namespace pqk
