// The K best items of a pass over the catalogue that does something else with every score: lists of candidates.
//
// The items are taken in pieces, in the order of their ids.  Of the first piece every score goes to the position's list; of the
// others those above its floor, a score that `keep` earlier items reach.  Between the pieces select_kernel cuts the lists back to
// little more than `keep` keys and raises the floors.  A later item that only ties with the floor ranks behind those `keep`, so the test
// is z > floor: equal scores add nothing, and whatever order the scores come in, the result is right.
//
// A workgroup has a region of each of its positions' lists, as long as it has items, and counts in LDS what it puts there.  (Counters of all workgroups
// in memory took the longest part of a pass: 64 of them, 53,000 candidates, 280 us.)
#pragma once
#include <math.h>
#include "head_common.hpp"

namespace pqk {
namespace head {

constexpr int kBins = 2048;
constexpr int kGroups = 64, kFewKept = 40;           // see cut_to_few()
constexpr int kMostKept = 1024;                      // keys that a cut leaves at most
constexpr int kMostRegions = 2048;                   // workgroups that share the items of a piece
// Keys that a thread of a cut holds; where a list has more each pass reads them again.  (kMostKeys by 1024 threads: 30,000 items of 128, 10 positions, K = 10, 30.4 and, held, 20.3 us; by
// 256, whose registers then leave a compute unit fewer workgroups, 400 positions of 25,000 59.5 and 60.9.)
constexpr int kFewKeys = 4, kManyKeys = 16, kMostKeys = 32;

struct Lists {
    uint64_t* keys;            // [B][cap]: all keys of the first piece, or the regions of a later one
    int* counts;               // [B][kMostRegions]: a position's side by side, which a cut reads
    uint64_t* kept;            // [B][kMostKept]: of the pieces before
    int* kept_count;           // [B]
    float* floor;              // [B]
    long long cap;
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

// A candidate to the workgroup's region, which begins at `region` and counts in *count (LDS).
__device__ __forceinline__ void append(const Lists& l, int q, long long region, int* count, float z, uint32_t item) {
    l.keys[(size_t)q * l.cap + region + atomicAdd(count, 1)] = key_of(z, item);       // (what order a region is in changes no result)
}

// A cut is made by a workgroup of 1024 threads, or of 256 where there are positions enough to give a compute unit several.
template <int THREADS>
struct SelectMemory {
    alignas(16) uint32_t histogram[kBins];
    alignas(16) uint32_t tops[kGroups];
    int begin[kMostRegions];                         // where a region's keys begin among all of them
    uint64_t part[THREADS / kWave][2];
    uint32_t sums[THREADS / kWave];
    int above, taken, chosen, count;
    uint32_t low;
    uint64_t least;
};

// What lies before the thread's own value among those of all threads.
template <int THREADS>
__device__ __forceinline__ uint32_t sums_before(uint32_t own, SelectMemory<THREADS>& mem, uint32_t& all) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    uint32_t sum = own;
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) {
        const uint32_t v = __shfl_up(sum, x);
        if (lane >= x) sum += v;
    }
    if (lane == kWave - 1) mem.sums[wave] = sum;
    __syncthreads();
    uint32_t before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) {
        const uint32_t v = mem.sums[w];
        if (w < wave) before += v;
        all += v;
    }
    return before + sum - own;
}

// The keys of a position's list: those kept, then the regions' (a list without regions: `kept` alone).
struct Keys {
    const uint64_t *kept, *keys;
    const int* begin;
    long long region;
    int kept_n, regions, n;
    __device__ __forceinline__ uint64_t operator()(int i) const {
        if (i < kept_n) return kept[i];
        int first = 0, count = regions;                          // (the last region that begins at i or before)
        while (count > 1) {
            const int half = count / 2;
            const bool there = begin[first + half] <= i;
            first = there ? first + half : first;
            count = there ? count - half : half;
        }
        return keys[first * region + (i - begin[first])];
    }
};

// A list's keys as a cut's passes meet them: R a thread in registers, or each from where it lies.
template <int THREADS, int R>
struct HeldKeys {
    uint64_t k[R];
    int n, own;                                                // of the list, of the thread
    __device__ __forceinline__ HeldKeys(const Keys& all) : n(all.n), own(0) {
        typedef uint64_t Pair __attribute__((ext_vector_type(2), aligned(8)));
        if (all.regions == 0) {
#pragma unroll
            for (int r = 0; r < R; r += 2) {
                const int i = 2 * ((int)threadIdx.x + r / 2 * THREADS);
                Pair two = {0, 0};
                own += min(max(n - i, 0), 2);
                if (i + 1 < n) two = *reinterpret_cast<const Pair*>(all.kept + i);
                else if (i < n) two[0] = all.kept[i];
                k[r] = two[0];
                k[r + 1] = two[1];
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int i = (int)threadIdx.x + r * THREADS;
                own += i < n;
                k[r] = i < n ? all(i) : 0;
            }
        }
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < own) f(k[r]);
    }
};
template <int THREADS>
struct FarKeys {
    const Keys& all;
    int n;
    __device__ __forceinline__ FarKeys(const Keys& keys) : all(keys), n(keys.n) {}
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        for (int i = threadIdx.x; i < n; i += THREADS) f(all(i));
    }
};

// A key that at least `keep` of the keys, and no more than `most` (over `keep`) of them, reach; 0 if there are no more than `keep`.  By histograms of 2048
// bins over the range that is left, each pass a look at all keys: one or two in the usual case, six at most (keys differ).
template <int THREADS, typename H>
__device__ __forceinline__ uint64_t cut(const H& held, int keep, int most, SelectMemory<THREADS>& mem) {
    constexpr int kWaves = THREADS / kWave, kOwn = kBins / THREADS;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    if (held.n <= keep) return 0;
    // The range to look in: up to the largest key, and from the least of the largest keys that groups of lanes have, if there are `keep` groups, which
    // hold a key each.  (Counted over the whole range, most of a long list's keys would queue up at a few bins.)
    const int group = held.n < THREADS ? 1 : keep <= THREADS / 64 ? 64 : keep <= THREADS / 16 ? 16 : keep <= THREADS / 4 ? 4 : 1;
    uint64_t low = 0, high = 0;
    const bool grouped = held.n >= THREADS && keep <= THREADS;
    if (!grouped) low = ~0ull;
    held.each([&](uint64_t k) {
        if (!grouped) low = k < low ? k : low;
        high = k > high ? k : high;
    });
#pragma unroll
    for (int i = 0; i < kOwn; ++i) mem.histogram[tid + i * THREADS] = 0;
    if (grouped) low = high;
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) {
        const uint64_t l = __shfl_xor(low, x), h = __shfl_xor(high, x);
        low = grouped && x < group ? (l > low ? l : low) : (l < low ? l : low);
        high = h > high ? h : high;
    }
    if (lane == 0) { mem.part[wave][0] = low; mem.part[wave][1] = high; }
    __syncthreads();
    low = mem.part[lane % kWaves][0];
    high = mem.part[lane % kWaves][1];
#pragma unroll
    for (int x = 1; x < kWaves; x *= 2) {
        const uint64_t l = __shfl_xor(low, x), h = __shfl_xor(high, x);
        low = l < low ? l : low;
        high = h > high ? h : high;
    }
    int above = 0;                                                // keys over the range
    while (true) {
        const int bits = 64 - __clzll((long long)((high - low) | 1)), shift = bits > 11 ? bits - 11 : 0;
        held.each([&](uint64_t k) {
            if (k >= low && k <= high) atomicAdd(&mem.histogram[(uint32_t)((k - low) >> shift)], 1u);
        });
        __syncthreads();
        // thread t has the bins from kBins - 1 - kOwn t downwards: what lies over them by a scan
        uint32_t bin[kOwn], sum = 0, all;
        const int top = kBins - 1 - kOwn * tid;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            bin[i] = mem.histogram[top - i];
            mem.histogram[top - i] = 0;
            sum += bin[i];
        }
        uint32_t begin = (uint32_t)above + sums_before(sum, mem, all);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            if (begin < (uint32_t)keep && begin + bin[i] >= (uint32_t)keep) {       // (one bin of one thread: the keep-th key is in it)
                mem.chosen = top - i;
                mem.above = (int)begin;
                mem.taken = (int)(begin + bin[i]);
            }
            begin += bin[i];
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
__host__ __device__ constexpr int most_of(int keep) { return keep + keep / 4 + 32 < kMostKept ? keep + keep / 4 + 32 : kMostKept; }

// A list's `keep` largest keys, where these are few (kFewKept: 63 to be expected), without histograms: of the largest scores of 64 groups of keys (those that come to a
// lane's number in all waves) the keep-th largest is one that `keep` keys reach, and little more do: 64 ln(64 / (64 - keep)) are to be expected.  These come to LDS and are
// put in order.  mem.tops holds the groups' largest, with the group's number for the last bits, so that no two are the same.
// Returns whether they were few enough (of equal scores there may be more); then out[] is in order.
// 10,000 keys, 10 of them kept: 2 us of the finish less than by histograms.  (256 groups for up to 140 kept took 2 us off 10,000 keys of one position, and cost 300 positions, whose
// lists keep the lanes busy, 5.)
constexpr int kFewTaken = 256;
template <int THREADS, typename H>
__device__ __forceinline__ bool cut_to_few(const H& held, int keep, uint64_t* out, SelectMemory<THREADS>& mem) {
    const int tid = threadIdx.x;
    uint64_t* taken = reinterpret_cast<uint64_t*>(mem.histogram);
    if (tid < kGroups) {
        const uint32_t own = mem.tops[tid];
        int above = 0;
#pragma unroll
        for (int i = 0; i < kGroups / 4; ++i) {
            const uint4 t = reinterpret_cast<const uint4*>(mem.tops)[i];
            above += (t.x > own) + (t.y > own) + (t.z > own) + (t.w > own);
        }
        if (above == keep - 1) mem.low = own & ~(kGroups - 1u);
    }
    __syncthreads();
    const uint64_t low = (uint64_t)mem.low << 32;
    held.each([&](uint64_t k) {
        if (k >= low) {
            const int at = atomicAdd(&mem.count, 1);
            if (at < kFewTaken) taken[at] = k;
        }
    });
    __syncthreads();
    const int n = mem.count;
    if (n > kFewTaken) {
        __syncthreads();
        if (tid == 0) mem.count = 0;
        return false;
    }
    if (tid < n) {
        const uint64_t mine = taken[tid];
        int rank = 0;
#pragma unroll 8                                               // (their reads of LDS on their way together)
        for (int i = 0; i < n; ++i) rank += taken[i] > mine;
        if (rank < keep) out[rank] = mine;
        if (rank == keep - 1) mem.least = mine;
    }
    return true;
}

// Cuts a position's list: what is left in out[] (in order, or in none: `sorted`), `keep` at least (or all) and most_of(keep) at most; returns how many, and in `least` what
// they reach (0: as good as nothing was cut).  last: no floor is asked for.  stored: how many keys the first piece left, if that was the last piece; else regions of `region` keys each.
// meanwhile() is called while the keys are on their way, and after a barrier aside(), while the first wave (of the others little is asked) looks for the cut.
template <int THREADS, typename Meanwhile, typename Aside>
__device__ __forceinline__ int cut_list(const Lists& l, int q, int stored, int regions, long long region, bool last, uint64_t* out, bool& sorted, uint64_t& least, SelectMemory<THREADS>& mem,
                                        Meanwhile meanwhile, Aside aside) {
    const int tid = threadIdx.x, most = last ? l.keep + 16 : most_of(l.keep);       // (of the last every key is scored again)
    const uint64_t* keys = l.keys + (size_t)q * l.cap;
    Keys all{l.kept + (size_t)q * kMostKept, keys, mem.begin, region, stored, 0, stored};
    if (stored) all.kept = keys;
    else {
        all.kept_n = l.kept_count[q];
        all.regions = regions;
        constexpr int kOwn = kMostRegions / THREADS;
        int own[kOwn], sum = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            own[i] = kOwn * tid + i < regions ? l.counts[(size_t)q * kMostRegions + kOwn * tid + i] : 0;
            sum += own[i];
        }
        uint32_t total;
        int before = all.kept_n + (int)sums_before((uint32_t)sum, mem, total);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            mem.begin[kOwn * tid + i] = before;
            before += own[i];
        }
        all.n = all.kept_n + (int)total;
    }
    if (tid < kGroups) mem.tops[tid] = 0;
    if (tid == 0) mem.count = 0;
    __syncthreads();
    int left = 0;
    auto run = [&](const auto& held) {
        meanwhile();
        const bool any = held.n > (last ? most : l.keep), few = any && l.keep <= kFewKept;
        if (few) {
            uint32_t top = 0;
            held.each([&](uint64_t k) { top = max(top, (uint32_t)(k >> 32)); });
            atomicMax(&mem.tops[tid % kGroups], (top & ~(kGroups - 1u)) | (uint32_t)(tid % kGroups));
        }
        __syncthreads();
        aside();
        sorted = few && cut_to_few<THREADS>(held, l.keep, out, mem);
        if (!sorted) {
            least = any ? cut<THREADS>(held, l.keep, most, mem) : 0;
            held.each([&](uint64_t k) {
                if (k >= least) out[atomicAdd(&mem.count, 1)] = k;
            });
        }
        __syncthreads();
        left = mem.count;
        if (sorted) { left = l.keep; least = mem.least; }
    };
    if (all.n <= kFewKeys * THREADS) run(HeldKeys<THREADS, kFewKeys>(all));
    else if (all.n <= kManyKeys * THREADS) run(HeldKeys<THREADS, kManyKeys>(all));
    else if (THREADS == 1024 && all.n <= kMostKeys * THREADS) run(HeldKeys<THREADS, THREADS == 1024 ? kMostKeys : kManyKeys>(all));
    else run(FarKeys<THREADS>(all));
    return left;
}

// grid = positions: cuts the lists between two pieces and sets the floors.  Chains of latencies again: 6 to 10 us for 203 positions of 10 + 16 keys or 512 of 100, 9 to 15 for 1024 of 116.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void select_kernel(Lists l, int stored, int regions, long long region) {
    __shared__ SelectMemory<THREADS> mem;
    __shared__ uint64_t out[kMostKept];
    const int q = blockIdx.x, tid = threadIdx.x;
    uint64_t least;
    bool sorted;
    const int n = cut_list(l, q, stored, regions, region, false, out, sorted, least, mem, [] {}, [] {});
    for (int i = tid; i < n; i += THREADS) l.kept[(size_t)q * kMostKept + i] = out[i];
    if (tid == 0) {
        l.kept_count[q] = n;
        if (least != 0) l.floor[q] = score_of(least);          // (a list of `keep` keys, of which nothing is cut, has the floor that it had)
    }
}

// ---------------------------------------------------------------------------------------------------------------
// host side

inline bool many_lists(int B) { return B > kCUs; }

// The pieces of a pass over N items: `first` items, whose scores are all stored, then as many as the lists have room for and no more than `growth`
// times the items before them: a list gets some growth * keep new keys in each.  How many pieces: a cut and what it stops take some 25 us, a candidate 25 to 150 ps over the chip (1024
// positions, 116 kept, 840,000 candidates beside 262,144 items of 512 bfloat16 46 us; 512 positions by sub-ids, K = 100, counted at 25 547 us, at 50, which makes a piece more, 556).
// `most`: of the candidates of a piece, where more than that take much longer each.
// The lists of a piece, the only one among them, take kListBytes, or what `least` items take of so many positions (8192 of 65,535: 4.3 GB).
constexpr long long kOnePiece = 16384, kListBytes = 1LL << 31;
struct Passes {
    long long N, first, room, growth;
    int keep;
    long long after(long long done) const {                      // items of the piece after `done` items
        if (done == 0) return first;
        const long long most = done * growth < room ? done * growth : room;
        const long long n = most > 16384 ? most / 16384 * 16384 : most;          // (whole rounds of 256 x 256 tiles over the chip)
        return n < N - done ? n : N - done;
    }
};
inline Passes passes_of(long long N, int B, int keep, double most = 1e300) {
    Passes p{N, N, N, 1, (int)(keep < N ? keep : N)};
    if (keep == 0) return p;
    const long long least = B <= 128 ? kOnePiece : (long long)round_up(8 * (size_t)keep, 4096);
    p.room = kListBytes / 8 / B;
    if ((N > kOnePiece && N > 2 * least) || (N > p.room && N > least)) p.first = least;
    if (p.room < p.first) p.room = p.first;
    double best = 1e300;
    for (int pieces = 1; pieces <= 8; ++pieces) {
        const double growth = pow((double)N / (double)p.first, 1.0 / pieces), candidates = (double)B * keep * growth, cost = pieces * (25.0 + 2.5e-5 * candidates);
        if (cost < best || (double)B * keep * (double)p.growth > most) { best = cost; p.growth = (long long)ceil(growth); }
    }
    return p;
}

// Where the sums of a piece's groups go, among a position's `slots`: behind those of the pieces before, or, where these would take more than kSumBytes (one position has some hundred
// groups in a piece, 65,535 have a hundred pieces a million items), in their places, joined with what is there.
constexpr size_t kSumBytes = (size_t)64 << 20;
struct Sums {
    int slots = 0, most = 0;
    bool joined = false;
    void piece(int groups) { slots += groups; most = groups > most ? groups : most; }
    void lay_out(int B) {
        joined = (size_t)slots * B * sizeof(float4) > kSumBytes;
        if (joined) slots = most;
    }
    size_t bytes(int B) const { return (size_t)slots * B * sizeof(float4); }
    // after a piece of so many groups: where the next one's sums go, and how many places there hold sums already
    void advance(int groups, int& done, int& written) const {
        if (joined) written = groups > written ? groups : written;
        else done += groups;
    }
};

// Where the lists lie in a workspace, behind `at` bytes.
struct ListLayout {
    long long cap = 0;
    size_t keys_at, counts_at, kept_at, kept_count_at, floor_at, bytes;
    void piece(long long keys) { cap = keys > cap ? keys : cap; }     // a piece whose regions take so many keys
    void lay_out(size_t at, int B, const Passes& p) {
        const size_t lists = p.keep ? B : 0, on = p.first < p.N ? lists : 0;             // (one piece is cut at the end alone, from where its keys lie)
        keys_at = round_up(at, 256);
        counts_at = keys_at + round_up(lists * cap * sizeof(uint64_t), 256);
        kept_at = counts_at + round_up(on * kMostRegions * sizeof(int), 256);
        kept_count_at = kept_at + round_up(on * kMostKept * sizeof(uint64_t), 256);
        floor_at = kept_count_at + round_up(on * sizeof(int), 256);
        bytes = floor_at + round_up(on * sizeof(float), 256);
    }
    Lists lists(unsigned char* ws, int keep) const {
        return Lists{reinterpret_cast<uint64_t*>(ws + keys_at), reinterpret_cast<int*>(ws + counts_at), reinterpret_cast<uint64_t*>(ws + kept_at),
                     reinterpret_cast<int*>(ws + kept_count_at), reinterpret_cast<float*>(ws + floor_at), cap, keep};
    }
};

inline hipError_t launch_select(const Lists& l, int B, int stored, int regions, long long region, hipStream_t st) {
    if (many_lists(B)) hipLaunchKernelGGL(select_kernel<256>, dim3(B), dim3(256), 0, st, l, stored, regions, region);
    else hipLaunchKernelGGL(select_kernel<1024>, dim3(B), dim3(1024), 0, st, l, stored, regions, region);
    return hipGetLastError();
}

}  // namespace head
}  // namespace pqk
