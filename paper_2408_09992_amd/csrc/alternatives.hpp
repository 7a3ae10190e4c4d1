// The K best items of a pass over the catalogue that does something else with every score: lists of candidates.
//
// The items are taken in pieces, in the order of their ids.  Of the first piece every score goes to the position's list; of the
// others those above its floor, a score that `keep` earlier items reach.  Between the pieces select_kernel cuts the lists back to
// little more than `keep` keys and raises the floors.  A later item that only ties with the floor ranks behind those `keep`, so the test
// is z > floor: no order of the scores makes a list overflow that holds what was kept and a piece, and equal scores add nothing.
#pragma once
#include "head_common.hpp"

namespace pqk {
namespace head {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / kWave;
constexpr int kMostKept = 1024;                      // keys that a cut leaves at most

struct Lists {
    uint64_t* keys;            // [B][cap]
    int* count;                // [B]
    float* floor;              // [B]
    uint32_t cap;
    int keep;                  // 0: no alternatives are asked for
};

// Keys in the order of TopK: score descending, then id ascending, is the key descending.  -0 ranks as +0, a NaN behind everything.
__device__ __forceinline__ uint64_t key_of(float z, uint32_t item) {
    const uint32_t u = __builtin_bit_cast(uint32_t, z + 0.0f);
    const uint32_t order = z != z ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
    return (uint64_t)order << 32 | (uint32_t)~item;
}
__device__ __forceinline__ uint32_t item_of(uint64_t key) { return ~(uint32_t)key; }
__device__ __forceinline__ float score_of(uint64_t key) {
    const uint32_t order = (uint32_t)(key >> 32);
    if (order <= 0x007FFFFFu) return -__builtin_inff();           // (also what ranked as a NaN)
    return __builtin_bit_cast(float, (order & 0x80000000u) ? order & 0x7FFFFFFFu : ~order);
}
__device__ __forceinline__ void append(const Lists& l, int q, float z, uint32_t item) {
    const int at = atomicAdd(l.count + q, 1);                     // (what order the lists are in changes no result)
    if ((uint32_t)at < l.cap) l.keys[(size_t)q * l.cap + at] = key_of(z, item);
}

struct SelectMemory {
    uint32_t histogram[2048];
    uint64_t part[kSelectWaves][2];
    uint32_t sums[kSelectWaves];
    uint64_t low, high;
    int above, taken, chosen;
};

// A key that at least `keep` of keys[0 .. n - 1], and no more than `most` (most > keep), reach; 0 if n <= keep.  By histograms of 2048 bins over
// the range that is left, each pass a look at all keys: one or two in the usual case, six at most (keys differ).
__device__ __forceinline__ uint64_t cut(const uint64_t* keys, int n, int keep, int most, SelectMemory& mem) {
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    if (n <= keep) return 0;
    uint64_t low = ~0ull, high = 0;
    for (int i = tid; i < n; i += kSelectThreads) {
        const uint64_t k = keys[i];
        low = k < low ? k : low;
        high = k > high ? k : high;
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) {
        const uint64_t l = __shfl_xor(low, x), h = __shfl_xor(high, x);
        low = l < low ? l : low;
        high = h > high ? h : high;
    }
    if (lane == 0) { mem.part[wave][0] = low; mem.part[wave][1] = high; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
        low = mem.part[w][0] < low ? mem.part[w][0] : low;
        high = mem.part[w][1] > high ? mem.part[w][1] : high;
    }
    int above = 0;                                                // keys over the range
    while (true) {
        const int bits = 64 - __clzll((long long)(high - low | 1)), shift = bits > 11 ? bits - 11 : 0;
        mem.histogram[tid] = 0;
        mem.histogram[tid + 1024] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kSelectThreads) {
            const uint64_t k = keys[i];
            if (k >= low && k <= high) atomicAdd(&mem.histogram[(uint32_t)((k - low) >> shift)], 1u);
        }
        __syncthreads();
        // thread t has the bins 2047 - 2t and 2046 - 2t: what lies over them by a scan
        const uint32_t upper = mem.histogram[2047 - 2 * tid], lower = mem.histogram[2046 - 2 * tid];
        uint32_t sum = upper + lower;
#pragma unroll
        for (int x = 1; x < kWave; x *= 2) {
            const uint32_t v = __shfl_up(sum, x);
            if (lane >= x) sum += v;
        }
        if (lane == kWave - 1) mem.sums[wave] = sum;
        __syncthreads();
        uint32_t before = (uint32_t)above;
        for (int w = 0; w < wave; ++w) before += mem.sums[w];
        const uint32_t end = before + sum, begin = end - upper - lower;
        if (begin < (uint32_t)keep && end >= (uint32_t)keep) {    // (one thread: the keep-th key is in its bins)
            const bool first = begin + upper >= (uint32_t)keep;
            mem.chosen = first ? 2047 - 2 * tid : 2046 - 2 * tid;
            mem.above = (int)(first ? begin : begin + upper);
            mem.taken = (int)(first ? begin + upper : end);
        }
        __syncthreads();
        low += (uint64_t)mem.chosen << shift;
        above = mem.above;
        const int taken = mem.taken;
        if (taken <= most || shift == 0) return low;
        const uint64_t last = low + ((1ull << shift) - 1);
        high = last < high ? last : high;
        __syncthreads();
    }
}

// How many keys a cut to `keep` may leave: a few more save a pass.
__device__ __forceinline__ int most_of(int keep) { return min(kMostKept, keep + keep / 4 + 32); }

// grid = positions.  stored: how many keys the first piece left, or 0: the counts say.  Leaves kept keys, their count and the floor.
template <int>                                        // (a template: only what launches it has it)
__global__ __launch_bounds__(kSelectThreads) void select_kernel(Lists l, int stored) {
    __shared__ SelectMemory mem;
    __shared__ uint64_t kept[kMostKept];
    __shared__ int count;
    const int q = blockIdx.x, tid = threadIdx.x;
    uint64_t* keys = l.keys + (size_t)q * l.cap;
    const int n = stored ? stored : min(l.count[q], (int)l.cap);
    if (tid == 0) count = 0;
    const uint64_t least = cut(keys, n, l.keep, most_of(l.keep), mem);
    __syncthreads();
    for (int i = tid; i < n; i += kSelectThreads) {
        const uint64_t k = keys[i];
        if (k >= least) kept[atomicAdd(&count, 1)] = k;
    }
    __syncthreads();
    for (int i = tid; i < count; i += kSelectThreads) keys[i] = kept[i];
    if (tid == 0) {
        l.count[q] = count;
        l.floor[q] = score_of(least);
    }
}

// The last cut: the keys that are left, in kept[]; returns how many, `keep` (or all) at least and kMostKept at most.
__device__ __forceinline__ int last_cut(const Lists& l, int q, int stored, uint64_t* kept, int& count, SelectMemory& mem) {
    const int tid = threadIdx.x;
    const uint64_t* keys = l.keys + (size_t)q * l.cap;
    const int n = stored ? stored : min(l.count[q], (int)l.cap), most = most_of(l.keep);
    if (tid == 0) count = 0;
    const uint64_t least = n <= most ? 0 : cut(keys, n, l.keep, most, mem);
    __syncthreads();
    for (int i = tid; i < n; i += kSelectThreads) {
        const uint64_t k = keys[i];
        if (k >= least) kept[atomicAdd(&count, 1)] = k;
    }
    __syncthreads();
    return count;
}

// ---------------------------------------------------------------------------------------------------------------
// host side

// The pieces of a pass over N items: `first` items, whose scores are all stored, then as many as the lists have room for and no more than kGrowth
// times the items before them, so that a list gets some kGrowth * keep new keys.
constexpr long long kOnePiece = 16384, kGrowth = 32, kListBytes = 1LL << 31;
struct Passes {
    long long N, first, cap;
    int keep;
    long long after(long long done) const {                      // items of the piece after `done` items
        if (done == 0) return first;
        long long n = done * kGrowth < cap - kMostKept ? done * kGrowth : cap - kMostKept;
        return n < N - done ? n : N - done;
    }
    size_t key_bytes(int B) const { return keep ? round_up((size_t)B * cap * sizeof(uint64_t), 256) : 0; }
};
inline Passes pieces_of(long long N, int B, int keep) {
    Passes p{N, N, 0, (int)(keep < N ? keep : N)};
    if (keep == 0) return p;
    const long long least = (long long)round_up(8 * (size_t)keep, 4096);
    if (N > kOnePiece && N > 2 * least) p.first = least;
    p.cap = N;
    if (p.first < N) {
        const long long room = kListBytes / 8 / B, need = p.first + 2 * kMostKept;
        p.cap = room > need ? room : need;
        if (p.cap > N + kMostKept) p.cap = N + kMostKept;
    }
    return p;
}

inline hipError_t launch_select(const Lists& l, int B, int stored, hipStream_t st) {
    hipLaunchKernelGGL(select_kernel<0>, dim3(B), dim3(kSelectThreads), 0, st, l, stored);
    return hipGetLastError();
}

}  // namespace head
}  // namespace pqk
