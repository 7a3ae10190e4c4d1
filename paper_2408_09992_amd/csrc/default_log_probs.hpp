// Log-probabilities of given items, entropy and the likeliest items by the default scorer's W phi (pq_default_log_probs): the cross entropy's pass
// over W (default_cross_entropy.hpp) with one more sum, and with candidates for the K best (alternatives.hpp).
//
//   r_qi = W[i] . phi_q   lse = log sum_i exp(r_i / T)   log p_i = r_i / T - lse   entropy = ln 2 (log2 s - t / s), s = sum 2^x, t = sum 2^x x, x = r log2 e / T - c
#pragma once
#include "pqtopk_probs.h"
#include "default_cross_entropy.hpp"
#include "alternatives.hpp"
#include "teacher.hpp"

namespace pqk {
namespace head {

struct DenseProbsArgs {
    const void *W, *H;
    long long N;
    int B, d;
    float scale;                                       // log2 e over the temperature
    long long first, end;                              // the piece's items
    int store;                                         // whether all its scores go to the lists
    long long item_tiles;
    int tiles_each, groups, position_tiles;
    float4* partial;                                   // [B][partials], of all pieces: (reference, sum, weighted sum); of this one from `done` on
    int partials, done, written;                       // of its places the first `written` hold earlier pieces' sums
    Lists lists;
    long long region;                                  // places of a region
};

// A group's region of a position's list is divided between the lanes that have scores of it (kShares of them), so that each counts its own in a register: a
// counter in LDS, whose answer every candidate waits for, took 180 us of the 1.9 ms of 1024 positions' best 100 of 1.28M items, where this takes 110.
template <typename Tile, int ITEMS> constexpr int kShares = ITEMS / (32 * Tile::MI) * 2;

// grid: groups of tiles of items x tiles of positions, one of which a chiplet takes one after the other (chiplet_order).  Bound by the matrix cores and the exponentials between the
// products: 262,144 items of 512 bfloat16 and 1024 positions 305 to 339 us on three cards, 811 to 900 TFLOP/s with the candidates (the loss alone 860 to 930).
template <typename T, int BN, int ITEMS>
__global__ __launch_bounds__((ScoresTile<T, BN, ITEMS>::kThreads), 2) void default_log_probs_kernel(DenseProbsArgs a) {
    using Tile = ScoresTile<T, BN, ITEMS>;
    constexpr int MI = Tile::MI, NI = Tile::NI, kRowWaves = ITEMS / (32 * MI);
    __shared__ float4 stat[kRowWaves][BN];
    int group, pt;
    chiplet_order(blockIdx.x, a.position_tiles, group, pt);
    if (group >= a.groups) return;
    const int lane = threadIdx.x % kWave;
    float c[NI], s[NI], t[NI], floor[NI];
    int listed[NI];
    const int share = Tile::wave_row() / (32 * MI) * 2 + lane / 32;
    const int q0 = pt * BN + Tile::wave_col() + lane % 32;
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
        c[ni] = kLowest; s[ni] = 0.0f; t[ni] = 0.0f;
        listed[ni] = 0;
        floor[ni] = __builtin_inff();
        if (a.lists.keep && !a.store && q0 + 32 * ni < a.B) floor[ni] = a.lists.floor[q0 + 32 * ni];
    }
    for (int i = 0; i < a.tiles_each; ++i) {
        const long long tile = (long long)group * a.tiles_each + i;
        if (tile >= a.item_tiles) break;
        const long long item0 = a.first + tile * ITEMS;
        f32x16 acc[MI][NI];
        Tile::run(Operand{a.W, (size_t)a.d * sizeof(T), item0, a.N, 0, a.d}, Operand{a.H, (size_t)a.d * sizeof(T), pt * BN, a.B, 0, a.d}, acc);
        const int left = left_of(a.end - item0 - Tile::wave_row(), 32 * MI);
        const long long mine = item0 + Tile::wave_row() + 4 * (lane / 32);
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) {
            __builtin_amdgcn_sched_barrier(0);                 // (one column after the other: the registers hold no two of them)
            float top = -__builtin_inff();
            if (left < 32 * MI) {
                stay_a_branch();
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (32 * mi + 8 * (e / 4) + e % 4 >= left - 4 * (lane / 32)) acc[mi][ni][e] = -__builtin_inff();
            }
            float tops[MI][4];                                 // (of four items each)
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int four = 0; four < 4; ++four) {
                    tops[mi][four] = fmaxf(fmaxf(acc[mi][ni][4 * four], acc[mi][ni][4 * four + 1]), fmaxf(acc[mi][ni][4 * four + 2], acc[mi][ni][4 * four + 3]));
                    top = fmaxf(top, tops[mi][four]);
                }
            if (a.store || __any(top > floor[ni])) {
                int q = q0 + 32 * ni;
                asm volatile("" : "+v"(q));                    // (so that no address is kept in registers for a branch that is rarely taken)
                uint64_t* keys = a.lists.keys + (size_t)q * a.lists.cap;
                if (a.store) keys += mine - a.first;
                else keys += ((size_t)group * kShares<Tile, ITEMS> + share) * a.region + listed[ni];
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int four = 0; four < 4; ++four) {
                        if (a.store) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int at = 32 * mi + 8 * four + e;
                                if (q < a.B && at < left - 4 * (lane / 32)) keys[at] = key_of(acc[mi][ni][4 * four + e], (uint32_t)(mine + at));
                            }
                        } else if (__any(tops[mi][four] > floor[ni])) {
                            stay_a_branch();
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (acc[mi][ni][4 * four + e] > floor[ni]) {
                                    *keys++ = key_of(acc[mi][ni][4 * four + e], (uint32_t)(mine + 32 * mi + 8 * four + e));
                                    ++listed[ni];
                                }
                        }
                    }
            }
            top *= a.scale;
            if (__any(top > c[ni] + kNearHeadroom)) {
                if (top > c[ni] + kNearHeadroom) raise_reference(c[ni], s[ni], t[ni], top);
            }
            float sum = 0.0f, sum_x = 0.0f;
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float x = fmaf(acc[mi][ni][e], a.scale, -c[ni]), p = exp2_fast(x);
                    sum += p;
                    sum_x = fmaf(p, x, sum_x);
                }
            if (__any(sum_x != sum_x)) {                       // (0 times -inf: a score that counts as -inf, rare enough to look for it here)
                stay_a_branch();
                sum_x = 0.0f;
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float x = fmaf(acc[mi][ni][e], a.scale, -c[ni]);
                        sum_x = weighted(exp2_fast(x), x, sum_x);
                    }
            }
            s[ni] += sum;
            t[ni] += sum_x;
        }
    }
    if (a.lists.keep && !a.store) {
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
            if (q0 + 32 * ni < a.B) a.lists.counts[(size_t)(q0 + 32 * ni) * kMostRegions + group * kShares<Tile, ITEMS> + share] = listed[ni];
    }
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
        join_sums(c[ni], s[ni], t[ni], __shfl_xor(c[ni], 32), __shfl_xor(s[ni], 32), __shfl_xor(t[ni], 32));
        if (lane < 32) stat[Tile::wave_row() / (32 * MI)][Tile::wave_col() + 32 * ni + lane] = make_float4(c[ni], s[ni], t[ni], 0.0f);
    }
    __syncthreads();
    const int q = pt * BN + threadIdx.x;
    if ((int)threadIdx.x < BN && q < a.B) {
        float4 v = stat[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < kRowWaves; ++w) join_sums(v.x, v.y, v.z, stat[w][threadIdx.x].x, stat[w][threadIdx.x].y, stat[w][threadIdx.x].z);
        float4& to = a.partial[(size_t)q * a.partials + a.done + group];
        if (group < a.written) join_sums(v.x, v.y, v.z, to.x, to.y, to.z);
        to = v;
    }
}

// The same for up to 64 positions of 16-bit operands, d <= 512: 64 positions, 1.3 GB of W, 221 us, 5.9 TB/s.
template <typename T, int D>
__global__ __launch_bounds__(kFewThreads, 2) void default_few_log_probs_kernel(DenseProbsArgs a) { few_sums<T, D, true>(a, a.first, a.end); }

struct DenseFinishArgs {
    const void *W, *H;
    const int* items;
    long long N;
    int B, d, n, K;
    double per_temperature, to_nats;                   // 1 / T; of log_sum64()
    const float4* partial;     // [B][groups], of all pieces
    int groups, stored, regions;                       // groups of all pieces; of the last piece what cut_list() takes
    long long region;
    Lists lists;
    float *log_probs, *entropy, *lse;
    int* top_items;
    float* top_log_probs;
};

// grid = positions: joins the groups' sums, scores the given items and the list's best in 64 bits, puts these in order.  A chain of latencies: one position 8.2 us; 1024 positions, whose
// 117 rows each come from memory as a rule, 40.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void default_log_probs_finish_kernel(DenseFinishArgs a) {
    __shared__ SelectMemory<THREADS> mem;
    __shared__ uint64_t kept[kMostKept];
    __shared__ double score[kMostKept];
    __shared__ float4 sums[THREADS / kWave];
    __shared__ double lse_of_all;
    constexpr int kWaves = THREADS / kWave;
    const int q = blockIdx.x, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    auto own_sums = [&] {
        float c = kLowest, s = 0.0f, t = 0.0f;
        for (int i = tid; i < a.groups; i += THREADS) {
            const float4 v = a.partial[(size_t)q * a.groups + i];
            join_sums(c, s, t, v.x, v.y, v.z);
        }
        if (wave * kWave < a.groups) join_wave(c, s, t);
        if (lane == 0) sums[wave] = make_float4(c, s, t, 0.0f);
    };
    auto aside = [&] {                                         // (64-bit logarithms, by one wave)
        if (wave != kWaves - 1) return;
        float4 v = sums[lane % kWaves];
        join_wave<kWaves>(v.x, v.y, v.z);
        if (lane == 0) {
            lse_of_all = log_sum64(v.x, v.y, a.to_nats);
            a.lse[q] = (float)lse_of_all;
            a.entropy[q] = entropy_of(v.y, v.z);
        }
    };
    const T *W = static_cast<const T*>(a.W), *h = static_cast<const T*>(a.H) + (size_t)q * a.d;
    uint64_t least;
    bool sorted;
    int n = 0;
    if (a.K) n = cut_list<THREADS>(a.lists, q, a.stored, a.regions, a.region, true, kept, sorted, least, mem, own_sums, aside);
    else {
        own_sums();
        __syncthreads();
        aside();
        __syncthreads();
    }
    const double lse = lse_of_all;
    auto log_prob = [&](double z) { return log_prob_of(z * a.per_temperature, lse); };
    // (the given items and the candidates at once: a row's way here is most of what either takes)
    score_rows<0, THREADS>(W, h, a.d, a.n + n,
                        [&](int i) {
                            const int item = i < a.n ? a.items[(size_t)q * a.n + i] : (int)item_of(kept[i - a.n]);
                            return item < a.N ? (long long)item : -1LL;
                        },
                        [&](int i, bool there, double z) {
                            if (i < a.n) a.log_probs[(size_t)q * a.n + i] = there ? log_prob(z) : 0.0f;
                            else score[i - a.n] = z;
                        });
    if (a.K == 0) return;
    __syncthreads();
    for (int at = tid; at < n; at += THREADS) {
        // (a NaN, of which no rank comes, is taken for the lowest)
        const double mine = score[at] == score[at] ? score[at] : -__builtin_inf();
        int rank = 0;
#pragma unroll 8                                               // (their reads of LDS on their way together)
        for (int i = 0; i < n; ++i) {
            const double other = score[i] == score[i] ? score[i] : -__builtin_inf();
            rank += (other > mine) | ((other == mine) & (kept[i] << 32 > kept[at] << 32));          // (the lower id's key is the larger)
        }
        if (rank < a.K) {
            a.top_items[(size_t)q * a.K + rank] = (int)item_of(kept[at]);
            a.top_log_probs[(size_t)q * a.K + rank] = log_prob(score[at]);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------
// host side, by type of the operands (a translation unit each)

// Shares of a group's region, by the tile that a plan takes (few positions' kernel does not divide it).
inline int shares_of(const DensePlan& p) {
    if (p.few) return 1;
    return p.loss_items == 64 || p.positions >= 128 ? 4 : 8;
}
static_assert(kShares<ScoresTile<__bf16, 64, 64>, 64> == 4 && kShares<ScoresTile<__bf16, 64, 256>, 256> == 8 && kShares<ScoresTile<__bf16, 128, 256>, 256> == 4 &&
              kShares<ScoresTile<__bf16, 256, 256>, 256> == 4, "as shares_of() has it");

template <typename T> hipError_t dense_probs(const DensePlan& p, const DenseProbsArgs& a, hipStream_t st);
template <typename T> hipError_t dense_probs_finish(const DenseFinishArgs& a, hipStream_t st);

#ifdef PQ_PROBS_INSTANCE
template <typename T, int POS, int ITEMS>
hipError_t launch_probs(const DensePlan& p, const DenseProbsArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((default_log_probs_kernel<T, POS, ITEMS>), dim3(grid_of(p.groups, p.position_tiles)), dim3(ScoresTile<T, POS, ITEMS>::kThreads), 0, st, a);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_few_probs(const DensePlan& p, const DenseProbsArgs& a, hipStream_t st) {
    const dim3 grid(p.groups), threads(kFewThreads);
    if (a.d > 256) hipLaunchKernelGGL((default_few_log_probs_kernel<T, 512>), grid, threads, 0, st, a);
    else if (a.d > 128) hipLaunchKernelGGL((default_few_log_probs_kernel<T, 256>), grid, threads, 0, st, a);
    else if (a.d > 64) hipLaunchKernelGGL((default_few_log_probs_kernel<T, 128>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((default_few_log_probs_kernel<T, 64>), grid, threads, 0, st, a);
    return hipGetLastError();
}
template <typename T>
hipError_t dense_probs(const DensePlan& p, const DenseProbsArgs& a, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (p.few) return launch_few_probs<T>(p, a, st);
    }
    return p.loss_items == 64 ? launch_probs<T, 64, 64>(p, a, st) : p.positions == 256 ? launch_probs<T, 256, 256>(p, a, st)
           : p.positions == 128 ? launch_probs<T, 128, 256>(p, a, st) : launch_probs<T, 64, 256>(p, a, st);
}
template <typename T>
hipError_t dense_probs_finish(const DenseFinishArgs& a, hipStream_t st) {
    if (many_lists(a.B)) hipLaunchKernelGGL((default_log_probs_finish_kernel<T, 256>), dim3(a.B), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((default_log_probs_finish_kernel<T, 1024>), dim3(a.B), dim3(1024), 0, st, a);
    return hipGetLastError();
}
template hipError_t dense_probs<PQ_PROBS_INSTANCE>(const DensePlan&, const DenseProbsArgs&, hipStream_t);
template hipError_t dense_probs_finish<PQ_PROBS_INSTANCE>(const DenseFinishArgs&, hipStream_t);
#endif

}  // namespace head
}  // namespace pqk
