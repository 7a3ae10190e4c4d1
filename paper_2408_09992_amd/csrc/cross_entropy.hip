// Softmax cross entropy of the catalogue by sub-ids (pq_cross_entropy*), and its gradient with respect to the score tables.
//
//   r_qi = sum_k S[q][k][G[i][k]]      lse_q = log sum_i exp r_qi      loss_q = lse_q - r_q,t
//   dS[q][k][j] = g_q ( sum_{i: G[i][k] = j} exp(r_qi - lse_q) - [G[t][k] = j] )
//
// A workgroup serves Q queries over a share of the items.  Their tables lie in LDS with the queries side by side, so one
// 16-byte read answers a sub-id for four queries; a lane takes an item with all Q queries.  The codes stream through once
// per group of queries (from L2 after the first).
#include <type_traits>
#include "pqtopk_train.h"
#include "head_common.hpp"

namespace pqk {
namespace head {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
// Items a lane holds at once (loss, gradient): as many as leave the registers of four waves a SIMD room.
template <int M> constexpr int units_of() { return M >= 64 ? 1 : M >= 32 ? 2 : 4; }
template <int M, typename CT> constexpr int units_back_of() { return M * (int)sizeof(CT) >= 32 ? 1 : 2; }
constexpr float kHeadroom = 40.0f;                   // (log2) how far a score may rise over a lane's reference before that moves
constexpr float kFixedBits = 30.0f;                  // probabilities are whole multiples of 2^-62: 30 bits and 32 more below them

// Table entries per split in LDS: a one-byte sub-id never runs past 256, a two-byte one is held below b.
template <typename CT> __device__ __forceinline__ int entries(int b) { return sizeof(CT) == 1 ? 256 : b; }

// One item's sub-ids in registers: M of them, of type CT.
template <int M, typename CT>
struct Row {
    static constexpr int kBytes = M * (int)sizeof(CT), kWords = (kBytes + 3) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const CT* codes, uint32_t item) {
        const unsigned char* p = reinterpret_cast<const unsigned char*>(codes) + (size_t)item * kBytes;
        if constexpr (kBytes == 2) w[0] = *reinterpret_cast<const uint16_t*>(p);
        else if constexpr (kBytes == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
        else if constexpr (kBytes == 8) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; }
        else {
#pragma unroll
            for (int i = 0; i < kBytes / 16; ++i) {
                const uint4 v = reinterpret_cast<const uint4*>(p)[i];
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        }
    }
    __device__ __forceinline__ uint32_t code(int k, uint32_t last) const {
        if constexpr (sizeof(CT) == 1) return (w[k / 4] >> (8 * (k % 4))) & 255u;
        else return min((w[k / 2] >> (16 * (k % 2))) & 65535u, last);
    }
};
// A row of one-byte sub-ids turned by `by` places: what was sub-id (k + by) % M is sub-id k.
template <int M>
__device__ __forceinline__ Row<M, uint8_t> turned(Row<M, uint8_t> r, uint32_t by) {
    constexpr int W = Row<M, uint8_t>::kWords;
#pragma unroll
    for (int x = 1; x < W; x *= 2) {
        const uint32_t move = 0u - (by / (4u * x) & 1u);       // (all ones or none: a select would become an array in scratch memory)
        Row<M, uint8_t> s;
#pragma unroll
        for (int i = 0; i < W; ++i) s.w[i] = r.w[i] ^ ((r.w[i] ^ r.w[(i + x) % W]) & move);
        r = s;
    }
    Row<M, uint8_t> s;
#pragma unroll
    for (int i = 0; i < W; ++i) s.w[i] = __builtin_amdgcn_alignbyte(r.w[(i + 1) % W], r.w[i], by % 4);
    return s;
}
// Any m: sub-ids are read one by one where they are used.
template <typename CT>
struct Row<0, CT> {
    const CT* p;
    __device__ __forceinline__ void load_at(const CT* codes, uint32_t item, int m) { p = codes + (size_t)item * m; }
    __device__ __forceinline__ uint32_t code(int k, uint32_t last) const { return sizeof(CT) == 1 ? (uint32_t)p[k] : min((uint32_t)p[k], last); }
};

template <int M, typename CT>
__device__ __forceinline__ void load_row(Row<M, CT>& r, const CT* codes, uint32_t item, int m) {
    if constexpr (M == 0) r.load_at(codes, item, m);
    else r.load(codes, item);
}

template <int Q>
__device__ __forceinline__ void read_queries(const float* p, float (&v)[Q]) {
    if constexpr (Q == 1) v[0] = *p;
    else if constexpr (Q == 2) { const float2 t = *reinterpret_cast<const float2*>(p); v[0] = t.x; v[1] = t.y; }
    else {
#pragma unroll
        for (int i = 0; i < Q / 4; ++i) {
            const float4 t = reinterpret_cast<const float4*>(p)[i];
            v[4 * i] = t.x; v[4 * i + 1] = t.y; v[4 * i + 2] = t.z; v[4 * i + 3] = t.w;
        }
    }
}

// r_qi of one item for Q queries: Eq. 5's chain.
template <int M, typename CT, int Q>
__device__ __forceinline__ void item_scores(const Row<M, CT>& row, const float* table, int m, int b, float (&z)[Q]) {
    const int E = entries<CT>(b);
    const uint32_t last = (uint32_t)E - 1u;
    auto add = [&](int k) {
        float v[Q];
        read_queries<Q>(table + (size_t)((uint32_t)k * (uint32_t)E + row.code(k, last)) * Q, v);
#pragma unroll
        for (int r = 0; r < Q; ++r) z[r] = k == 0 ? v[r] : z[r] + v[r];
    };
    if constexpr (M > 0) {
#pragma unroll
        for (int k = 0; k < M; ++k) add(k);
    } else {
        for (int k = 0; k < m; ++k) add(k);
    }
}

// Tables of Q queries to LDS, [k][j][q]; queries past the batch repeat its last one, sub-ids from b to E are 0.
template <typename CT, int Q>
__device__ __forceinline__ void fill_tables(float* table, const float* S, int q0, int B, int m, int b) {
    const int E = entries<CT>(b);
    const size_t per_query = (size_t)m * b;
    const float* src[Q];
#pragma unroll
    for (int r = 0; r < Q; ++r) src[r] = S + (size_t)min(q0 + r, B - 1) * per_query;
    for (int i = threadIdx.x; i < m * E; i += kThreads) {
        const int k = i / E, j = i - k * E;
        float v[Q];
#pragma unroll
        for (int r = 0; r < Q; ++r) v[r] = j < b ? src[r][(size_t)k * b + j] : 0.0f;
#pragma unroll
        for (int r = 0; r < Q; ++r) table[(size_t)i * Q + r] = v[r];
    }
}

// What one position's statistics make of it, by one wave: lse, and the loss with the target's score (its m sub-item scores are
// fetched by as many lanes at once).
__device__ __forceinline__ void finish_position(float c, float s, const void* codes, int code_bytes, const float* S, const int* targets,
                                                long long N, int m, int b, int q, float* loss, float* lse) {
    const int lane = threadIdx.x % kWave, t = targets[q];
    const float l = log_sum(c, s);
    const bool has = t >= 0 && t < N && l != -__builtin_inff();
    float z = 0.0f;
    if (has) {
        for (int k = lane; k < m; k += kWave) {
            const size_t at = (size_t)t * m + k;
            const uint32_t g = code_bytes == 1 ? (uint32_t)static_cast<const uint8_t*>(codes)[at] : (uint32_t)static_cast<const uint16_t*>(codes)[at];
            z += S[((size_t)q * m + k) * b + min(g, (uint32_t)b - 1u)];
        }
#pragma unroll
        for (int x = 1; x < kWave; x *= 2) z += __shfl_xor(z, x);
    }
    if (lane == 0) {
        lse[q] = l;
        loss[q] = has ? l - z : 0.0f;
    }
}

struct LossArgs {
    const void* codes;
    const float* S;
    const int* targets;
    long long N;
    int B, m, b;
    uint32_t share;            // items per workgroup
    float2* partial;           // [gridDim.x][B]: (reference, sum), where the items are shared
    float *loss, *lse;
};

// grid = (shares of the items, groups of Q queries).
// Per item and query: m LDS words, m - 1 additions, a fused multiply-add, an exponential and an addition.  Each lane keeps a
// reference c and sum s per query (total s 2^c); the reference moves only when a score passes it by 2^kHeadroom, which the
// sum's exponent has room for, so the usual step has no maximum to carry.
// Bound by the lookups in LDS: 1024 positions of 1.27M items, m = 8, 742 us, 0.044 cycles each and compute unit; 16 of 5M items,
// m = 16, whose registers (71 a lane) leave a compute unit one workgroup, 113 us, 0.054.
template <int M, typename CT, int Q>
__global__ __launch_bounds__(kThreads) void cross_entropy_kernel(LossArgs a) {
    constexpr int kUnits = units_of<M>();
    extern __shared__ __align__(16) unsigned char smem[];
    float* table = reinterpret_cast<float*>(smem);
    float2* stat = reinterpret_cast<float2*>(smem + (size_t)a.m * entries<CT>(a.b) * Q * sizeof(float));      // [kWaves][Q]
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int q0 = blockIdx.y * Q;
    const CT* codes = static_cast<const CT*>(a.codes);
    fill_tables<CT, Q>(table, a.S, q0, a.B, a.m, a.b);
    __syncthreads();

    const uint32_t lo = blockIdx.x * a.share, hi = (uint32_t)min((long long)lo + a.share, a.N);
    float c[Q], s[Q];
#pragma unroll
    for (int r = 0; r < Q; ++r) { c[r] = kLowest; s[r] = 0.0f; }

    auto step = [&](const Row<M, CT> (&row)[kUnits], uint32_t first, auto whole) {
        float z[kUnits][Q];
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            item_scores<M, CT, Q>(row[u], table, a.m, a.b, z[u]);
            if (!decltype(whole)::value && first + u * kThreads >= hi) {
#pragma unroll
                for (int r = 0; r < Q; ++r) z[u][r] = -__builtin_inff();
            }
        }
        bool rise = false;
        float top[Q];
#pragma unroll
        for (int r = 0; r < Q; ++r) {
            top[r] = z[0][r];
#pragma unroll
            for (int u = 1; u < kUnits; ++u) top[r] = fmaxf(top[r], z[u][r]);
            top[r] *= kLog2e;
            rise |= top[r] > c[r] + kHeadroom;
        }
        if (__any(rise)) {
#pragma unroll
            for (int r = 0; r < Q; ++r) {
                if (top[r] > c[r] + kHeadroom) raise_reference(c[r], s[r], top[r]);
            }
        }
#pragma unroll
        for (int r = 0; r < Q; ++r)
#pragma unroll
            for (int u = 0; u < kUnits; ++u) s[r] += exp2_fast(fmaf(z[u][r], kLog2e, -c[r]));
    };

    Row<M, CT> row[kUnits];
    const uint32_t last = (uint32_t)(a.N - 1), stride = kThreads * kUnits;
    auto load = [&](uint32_t first) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) load_row<M, CT>(row[u], codes, min(first + u * kThreads, last), a.m);
    };
    load(lo + threadIdx.x);
    for (uint32_t base = lo; base < hi; base += stride) {
        const uint32_t first = base + threadIdx.x;
        Row<M, CT> now[kUnits];
#pragma unroll
        for (int u = 0; u < kUnits; ++u) now[u] = row[u];
        load(min(first + stride, last));                       // (the next step's sub-ids arrive while this one's scores are summed)
        if (hi - base >= stride) step(now, first, std::true_type{});
        else step(now, first, std::false_type{});
    }

    // the lanes' sums, then the waves'
#pragma unroll
    for (int r = 0; r < Q; ++r) {
#pragma unroll
        for (int x = 1; x < kWave; x *= 2) {
            const float c2 = __shfl_xor(c[r], x), s2 = __shfl_xor(s[r], x);
            join_sums(c[r], s[r], c2, s2);
        }
        if (lane == 0) stat[wave * Q + r] = make_float2(c[r], s[r]);
    }
    __syncthreads();
    if (wave < Q && q0 + wave < a.B) {
        float2 t = stat[wave];
        for (int w = 1; w < kWaves; ++w) join_sums(t.x, t.y, stat[w * Q + wave].x, stat[w * Q + wave].y);
        const int q = q0 + wave;
        if (gridDim.x == 1) finish_position(t.x, t.y, a.codes, sizeof(CT), a.S, a.targets, a.N, a.m, a.b, q, a.loss, a.lse);
        else if (lane == 0) a.partial[(size_t)blockIdx.x * a.B + q] = t;
    }
}

// One wave per position joins the shares' sums: 4 us, a launch.
__global__ __launch_bounds__(kWave) void cross_entropy_join_kernel(LossArgs a, int shares, int code_bytes) {
    const int q = blockIdx.x, lane = threadIdx.x;
    float c = kLowest, s = 0.0f;
    for (int i = lane; i < shares; i += kWave) {
        const float2 t = a.partial[(size_t)i * a.B + q];
        join_sums(c, s, t.x, t.y);
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) {
        const float c2 = __shfl_xor(c, x), s2 = __shfl_xor(s, x);
        join_sums(c, s, c2, s2);
    }
    finish_position(c, s, a.codes, code_bytes, a.S, a.targets, a.N, a.m, a.b, q, a.loss, a.lse);
}

struct BackArgs {
    const void* codes;
    const float* S;
    const int* targets;
    const float *lse, *grad;
    long long N;
    int B, m, b;
    int kept;                  // table entries whose sums a workgroup keeps (the others are other workgroups': blockIdx.z)
    uint32_t share;
    uint64_t* partial;         // [gridDim.x][B][m][b], where the items are shared
    float* dS;
};

__device__ __forceinline__ bool has_target(const BackArgs& a, int q) {
    const int t = a.targets[q];
    return t >= 0 && t < a.N && a.lse[q] != -__builtin_inff();
}

// A table entry's sum of probabilities (multiples of 2^-62) to its gradient.
__device__ __forceinline__ float gradient_of(const BackArgs& a, uint64_t sum, int q, int k, int j, int code_bytes) {
    if (!has_target(a, q)) return 0.0f;
    const size_t at = (size_t)a.targets[q] * a.m + k;
    const int g = code_bytes == 1 ? (int)static_cast<const uint8_t*>(a.codes)[at] : (int)static_cast<const uint16_t*>(a.codes)[at];
    // (a position whose scores hold a NaN has lse = NaN, of which its probabilities' whole numbers know nothing)
    const double p = a.lse[q] == a.lse[q] ? (double)sum * 0x1p-62 - (g == j ? 1.0 : 0.0) : (double)a.lse[q];
    return (float)((double)a.grad[q] * p);
}

// grid = (shares of the items, groups of Q queries, ranges of table entries: one but for the largest tables, Q = C = 1).
// Scores as in the loss, p = exp(r - lse), then p is added to m places of the sums in LDS.  Those are 64-bit integers: the
// order in which lanes and waves add does not matter, and the chip adds integers in LDS at ~10 cycles a wave instruction
// where floats take ~190.  What bounds it is those additions: about 0.13 cycles each per compute unit, a lookup 0.04 (1024 positions
// of 1.27M items with popular sub-ids, m = 8: 2.88 ms, 0.17 for both; 64 of 1.28M: 217 us).
// Each sum lies in Q * C places side by side, P = Q C of them a row: at step s of an item, lane l adds the query of place
// s ^ (l % P).  So the lanes of one instruction spread over all banks whatever the sub-ids are, and a popular sub-id is
// met by a P-th of the lanes at a time.  With fewer than four queries the C places of a query are summed at the end.
// For the same reason neighbouring lanes start at different splits (one-byte sub-ids): a sub-id that a fifth of the items
// share is met by a lane or two of an instruction instead of a fifth of them.
template <int M, typename CT, int Q, int C>
__global__ __launch_bounds__(kThreads) void cross_entropy_backward_kernel(BackArgs a) {
    constexpr int P = Q * C, kUnitsBack = units_back_of<M, CT>();
    extern __shared__ __align__(16) unsigned char smem[];
    const int E = entries<CT>(a.b);
    unsigned long long* sums = reinterpret_cast<unsigned long long*>(smem);
    float* table = reinterpret_cast<float*>(smem + (size_t)a.kept * P * sizeof(uint64_t));
    const int q0 = blockIdx.y * Q;
    constexpr bool kRanges = P == 1;                           // (any other instance keeps all entries)
    const uint32_t e0 = kRanges ? blockIdx.z * a.kept : 0u, e1 = (uint32_t)min(a.m * E, (int)e0 + a.kept);
    const CT* codes = static_cast<const CT*>(a.codes);
    fill_tables<CT, Q>(table, a.S, q0, a.B, a.m, a.b);
    for (int i = threadIdx.x; i < a.kept * P; i += kThreads) sums[i] = 0;
    float at[Q];                                               // exp2(z log2e - at) is p 2^30
    bool any = false;
#pragma unroll
    for (int r = 0; r < Q; ++r) {
        const int q = min(q0 + r, a.B - 1);
        const bool live = q0 + r < a.B && has_target(a, q);
        at[r] = live ? a.lse[q] * kLog2e - kFixedBits : __builtin_inff();
        any |= live;
    }
    __syncthreads();

    const uint32_t lo = blockIdx.x * a.share, hi = (uint32_t)min((long long)lo + a.share, a.N);
    const uint32_t last = (uint32_t)(a.N - 1), stride = kThreads * kUnitsBack, last_code = (uint32_t)E - 1u;
    constexpr bool kTurned = sizeof(CT) == 1 && M >= 4 && M <= 32;          // (LDS holds all entries of these: no ranges)
    static_assert(!(kTurned && kRanges), "an entry outside the range is told by its split");
    const uint32_t turn = threadIdx.x % P, split_turn = kTurned ? threadIdx.x / P % (M > 0 ? M : 1) : 0u;
    // LDS address of the lane's first place of split k's sums, sub-id 0
    const uint32_t sums_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)sums + turn * 8u;
    auto split_at = [&](int k) {
        const uint32_t split = kTurned ? ((uint32_t)k + split_turn) % (uint32_t)(M > 0 ? M : 1) : (uint32_t)k;
        return sums_at + split * (uint32_t)E * (P * 8u);
    };
    auto step = [&](const Row<M, CT>& row, bool there, auto whole) {
        float z[Q], p[Q];
        item_scores<M, CT, Q>(row, table, a.m, a.b, z);
#pragma unroll
        for (int r = 0; r < Q; ++r) {
            p[r] = exp2_fast(fmaf(z[r], kLog2e, -at[r]));
            if (!decltype(whole)::value) p[r] = there ? p[r] : 0.0f;
        }
        // place s ^ turn holds query (s ^ turn) % Q: with C copies a lane adds each query once, in the copy turn / Q
#pragma unroll
        for (int x = 1; x < Q; x *= 2) {
            const bool swap = (turn & (uint32_t)x) != 0;
#pragma unroll
            for (int r = 0; r < Q; ++r) {
                if ((r & x) == 0) {
                    const float lo_v = p[r], hi_v = p[r | x];
                    p[r] = swap ? hi_v : lo_v;
                    p[r | x] = swap ? lo_v : hi_v;
                }
            }
        }
        unsigned long long fixed[Q];
#pragma unroll
        for (int r = 0; r < Q; ++r) {
            const uint32_t upper = (uint32_t)p[r];
            const uint32_t lower = (uint32_t)(__builtin_amdgcn_fractf(p[r]) * 0x1p32f);
            fixed[r] = ((unsigned long long)upper << 32) | lower;
        }
        Row<M, CT> mine = row;
        if constexpr (kTurned) mine = turned<M>(row, split_turn);
        auto add = [&](int k, uint32_t first) {
            const uint32_t code = mine.code(k, last_code);
            uint32_t place = first + code * (P * 8u);
            if constexpr (kRanges) {
                if ((uint32_t)k * (uint32_t)E + code - e0 >= e1 - e0) return;
            }
#pragma unroll
            for (int r = 0; r < Q; ++r) {
                auto* to = (unsigned long long*)(__attribute__((address_space(3))) unsigned long long*)(uintptr_t)(place ^ (r * 8u));
                __hip_atomic_fetch_add(to, fixed[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            }
        };
        if constexpr (M > 0) {
#pragma unroll
            for (int k = 0; k < M; ++k) add(k, split_at(k) - (kRanges ? e0 * 8u : 0u));
        } else {
            for (int k = 0; k < a.m; ++k) add(k, split_at(k) - (kRanges ? e0 * 8u : 0u));
        }
    };
    if (any) {
        Row<M, CT> row[kUnitsBack];
        auto load = [&](uint32_t first) {
#pragma unroll
            for (int u = 0; u < kUnitsBack; ++u) load_row<M, CT>(row[u], codes, min(first + u * kThreads, last), a.m);
        };
        load(lo + threadIdx.x);
        for (uint32_t base = lo; base < hi; base += stride) {
            const uint32_t first = base + threadIdx.x;
            Row<M, CT> now[kUnitsBack];
#pragma unroll
            for (int u = 0; u < kUnitsBack; ++u) now[u] = row[u];
            load(min(first + stride, last));
            if (M < 64 && hi - base >= stride) {
#pragma unroll
                for (int u = 0; u < kUnitsBack; ++u) step(now[u], true, std::true_type{});
            } else {
#pragma unroll
                for (int u = 0; u < kUnitsBack; ++u) step(now[u], first + u * kThreads < hi, std::false_type{});
            }
        }
    }
    __syncthreads();

#pragma unroll
    for (int r = 0; r < Q; ++r) {
        const int q = q0 + r;
        if (q >= a.B) break;
        for (uint32_t i = threadIdx.x; i < e1 - e0; i += kThreads) {
            const int k = (int)((e0 + i) / (uint32_t)E), j = (int)(e0 + i) - k * E;
            if (j >= a.b) continue;
            unsigned long long total = 0;
#pragma unroll
            for (int copy = 0; copy < C; ++copy) total += sums[i * P + copy * Q + r];
            const size_t out = ((size_t)q * a.m + k) * a.b + j;
            if (gridDim.x > 1) a.partial[(size_t)blockIdx.x * a.B * a.m * a.b + out] = total;
            else a.dS[out] = gradient_of(a, total, q, k, j, sizeof(CT));
        }
    }
}

// The shares' sums of every table entry, added and turned into gradients, by LEADS threads an entry, each of them every LEADS-th
// share (the sums are whole numbers: any order gives the same).  One thread alone would wait for many shares one after the
// other: 5M items, one position 85 us for the gradient with one, 27 with eight; with few shares eight have nothing to do.
constexpr int kJoinThreads = 256, kJoinLeads = 8;
template <int LEADS>
__global__ __launch_bounds__(kJoinThreads) void cross_entropy_backward_join_kernel(BackArgs a, int shares, int code_bytes) {
    constexpr int kEntries = kJoinThreads / LEADS;
    __shared__ uint64_t part[LEADS][kEntries];
    const size_t entries = (size_t)a.B * a.m * a.b;
    const size_t i = (size_t)blockIdx.x * kEntries + threadIdx.x % kEntries;
    const int lead = threadIdx.x / kEntries;
    uint64_t total = 0;
    if (i < entries) {
#pragma unroll 8
        for (int s = lead; s < shares; s += LEADS) total += a.partial[(size_t)s * entries + i];
    }
    if constexpr (LEADS > 1) {
        part[lead][threadIdx.x % kEntries] = total;
        __syncthreads();
#pragma unroll
        for (int l = 1; l < LEADS; ++l) total += part[l][threadIdx.x % kEntries];              // (the first thread of an entry has the whole)
    }
    if (lead != 0 || i >= entries) return;
    const size_t row = i / a.b;
    a.dS[i] = gradient_of(a, total, (int)(row / a.m), (int)(row % a.m), (int)(i - row * a.b), code_bytes);
}

// ---------------------------------------------------------------------------------------------------------------
// host side

struct Plan {
    int Q, C, groups, shares, kept, ranges;
    uint32_t share;
    size_t lds;
};

int entries_of(int b, int code_bytes) { return code_bytes == 1 ? 256 : b; }

// How many shares the items are cut into: the least time by the cycles that an item takes a workgroup (`item`), that a
// workgroup takes besides (`fixed`: tables in, sums out), and that the launch takes which joins more than one share.
constexpr double kJoinCycles = 8000;                            // 3.5 us, as measured
void cut_items(Plan& p, long long N, long long workgroups, long long slots, double item, double fixed) {
    double best = 1e300;
    p.shares = 1;
    const long long least = 2 * kThreads, most = N / least > 0 ? N / least : 1;
    for (long long s = 1; s <= most && s <= 4 * kCUs; ++s) {
        if (workgroups * s > 4 * slots && s > 1) break;
        const double cost = (double)ceil_div(workgroups * s, slots) * ((double)ceil_div(N, s) * item + fixed) + (s > 1 ? kJoinCycles : 0);
        if (cost < best * 0.98) { best = cost; p.shares = (int)s; }
    }
    p.share = (uint32_t)ceil_div(N, p.shares);
    p.shares = (int)ceil_div(N, p.share);
}

constexpr size_t kStatBytes = (size_t)kWaves * 8 * sizeof(float2);

bool plan_loss(Plan& p, long long N, int B, int m, int b, int code_bytes) {
    const size_t entry_floats = (size_t)m * entries_of(b, code_bytes);
    p.Q = B >= 3 ? 4 : B;
    while (p.Q > 1 && entry_floats * 4 * p.Q + kStatBytes > kMaxLds) p.Q /= 2;
    p.C = 1;
    p.kept = 0;
    p.ranges = 1;
    p.lds = entry_floats * 4 * p.Q + kStatBytes;
    if (p.lds > kMaxLds) return false;
    p.groups = (int)ceil_div(B, p.Q);
    // Two workgroups run on a compute unit where LDS holds the tables of both and its registers (64 a lane then) the rows, which those of 16
    // and 32 bytes are too long for.  (Counted as two, they came in two rounds of half the items: 1.28M items, m = 16, one position 19.4 us
    // instead of 15.0, 300,000 and 64 positions 46 instead of 36; 5M, m = 16, 16 positions 124 instead of 117.)
    const bool long_rows = m == 16 || (m == 8 && code_bytes == 2) || (m == 32 && code_bytes == 1);
    const bool two = p.lds <= kMaxLds / 2 && !long_rows;
    // a lookup takes a compute unit 0.04 cycles a query (0.08 for one query alone); tables come in at some 20 bytes a cycle
    cut_items(p, N, p.groups, (two ? 2 : 1) * kCUs, m * (p.Q == 1 ? 0.08 : 0.045 * p.Q), 2000 + p.lds / 20.0);
    return true;
}

bool plan_backward(Plan& p, long long N, int B, int m, int b, int code_bytes) {
    const size_t E = entries_of(b, code_bytes), tables = (size_t)m * E * 4;
    // queries side by side, then copies of the sums, as far as LDS goes; where one query's sums do not fit beside its table,
    // workgroups share the entries and each computes the scores
    const size_t sums = (size_t)m * E * 8;
    p.Q = B >= 3 ? 4 : B;
    while (p.Q > 1 && (tables + sums) * p.Q > kMaxLds) p.Q /= 2;
    p.C = 8 / p.Q;
    while (p.C > 1 && (tables + sums * p.C) * p.Q > kMaxLds) p.C /= 2;
    p.ranges = 1;
    p.kept = (int)(m * E);
    if (p.Q * p.C == 1 && tables + sums > kMaxLds) {
        if (tables + 1024 * 8 > kMaxLds) return false;
        p.ranges = (int)ceil_div(sums, kMaxLds - tables);
        p.kept = (int)ceil_div((long long)m * E, p.ranges);
    }
    p.lds = tables * p.Q + (size_t)p.kept * 8 * p.Q * p.C;
    p.groups = (int)ceil_div(B, p.Q);
    // an addition to a sum takes 0.13 cycles a query
    cut_items(p, N, (long long)p.groups * p.ranges, kCUs, m * (p.Q == 1 ? 0.25 : 0.17 * p.Q), 2000 + p.lds / 20.0);
    return true;
}

int check_shape(long long N, int B, int m, int b, int code_bytes) {
    if (N < 1 || B < 1 || m < 1 || b < 1 || b > (code_bytes == 1 ? 256 : 65536) || N >= 2147483648LL) return PQ_ERR_SHAPE;
    if (m > PQ_MAX_M || B > PQ_MAX_B || (long long)m * entries_of(b, code_bytes) > 36864) return PQ_ERR_UNSUPPORTED;
    return PQ_OK;
}

size_t loss_workspace(const Plan& p, int B) { return round_up((p.shares > 1 ? (size_t)p.shares * B * sizeof(float2) : 0) + 16, 16); }
size_t backward_workspace(const Plan& p, int B, int m, int b) {
    return round_up((p.shares > 1 ? (size_t)p.shares * B * m * b * sizeof(uint64_t) : 0) + 16, 16);
}

template <int M, typename CT, int Q>
hipError_t go_loss(const Plan& p, const LossArgs& a, hipStream_t st) {
    hipError_t e = allow_lds(cross_entropy_kernel<M, CT, Q>, p.lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((cross_entropy_kernel<M, CT, Q>), dim3(p.shares, p.groups), dim3(kThreads), p.lds, st, a);
    return hipGetLastError();
}
// Whether LDS holds the tables of Q queries and P sums an entry (one-byte sub-ids; with two bytes b decides at run time).
template <int M, typename CT>
constexpr bool fits(int Q, int P) { return sizeof(CT) == 2 || (size_t)M * 256 * (4 * Q + 8 * P) <= kMaxLds; }

template <int M, typename CT>
hipError_t go_loss_q(const Plan& p, const LossArgs& a, hipStream_t st) {
    if constexpr (fits<M, CT>(4, 0)) { if (p.Q == 4) return go_loss<M, CT, 4>(p, a, st); }
    if (p.Q == 2) return go_loss<M, CT, 2>(p, a, st);
    return go_loss<M, CT, 1>(p, a, st);
}

template <int M, typename CT, int Q, int C>
hipError_t go_backward(const Plan& p, const BackArgs& a, hipStream_t st) {
    hipError_t e = allow_lds(cross_entropy_backward_kernel<M, CT, Q, C>, p.lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((cross_entropy_backward_kernel<M, CT, Q, C>), dim3(p.shares, p.groups, p.ranges), dim3(kThreads), p.lds, st, a);
    return hipGetLastError();
}
// Whether a plan of the gradient can be Q queries with C copies: one-byte sub-ids of M splits take the most copies that fit.
template <int M, typename CT>
constexpr bool reached(int Q, int C) {
    return M == 0 || sizeof(CT) == 2 || (fits<M, CT>(Q, Q * C) && (Q * C == 8 || !fits<M, CT>(Q, 2 * Q * C))) || (M == 64 && Q * C == 1);
}
template <int M, typename CT>
hipError_t go_backward_q(const Plan& p, const BackArgs& a, hipStream_t st) {
    if constexpr (reached<M, CT>(4, 2)) { if (p.Q == 4 && p.C == 2) return go_backward<M, CT, 4, 2>(p, a, st); }
    if constexpr (reached<M, CT>(4, 1)) { if (p.Q == 4) return go_backward<M, CT, 4, 1>(p, a, st); }
    if constexpr (reached<M, CT>(2, 4)) { if (p.Q == 2 && p.C == 4) return go_backward<M, CT, 2, 4>(p, a, st); }
    if constexpr (reached<M, CT>(2, 2)) { if (p.Q == 2 && p.C == 2) return go_backward<M, CT, 2, 2>(p, a, st); }
    if constexpr (reached<M, CT>(2, 1)) { if (p.Q == 2) return go_backward<M, CT, 2, 1>(p, a, st); }
    if constexpr (reached<M, CT>(1, 8)) { if (p.C == 8) return go_backward<M, CT, 1, 8>(p, a, st); }
    if constexpr (reached<M, CT>(1, 4)) { if (p.C == 4) return go_backward<M, CT, 1, 4>(p, a, st); }
    if constexpr (reached<M, CT>(1, 2)) { if (p.C == 2) return go_backward<M, CT, 1, 2>(p, a, st); }
    if constexpr (reached<M, CT>(1, 1)) return go_backward<M, CT, 1, 1>(p, a, st);
    else return hipErrorInvalidValue;                          // (no plan asks for it)
}

template <typename CT>
int loss(const CT* codes, const float* S, const int* targets, long long N, int B, int m, int b, float* out, float* lse, void* ws,
         size_t ws_bytes, void* stream) {
    if (!codes || !S || !targets || !out || !lse || !ws) return PQ_ERR_NULL;
    int rc = check_shape(N, B, m, b, sizeof(CT));
    if (rc != PQ_OK) return rc;
    Plan p;
    if (!plan_loss(p, N, B, m, b, sizeof(CT))) return PQ_ERR_UNSUPPORTED;
    if (((uintptr_t)codes & 15) || ((uintptr_t)ws & 15) || (((uintptr_t)S | (uintptr_t)targets | (uintptr_t)out | (uintptr_t)lse) & 3)) return PQ_ERR_ALIGN;
    if (ws_bytes < loss_workspace(p, B)) return PQ_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    LossArgs a{codes, S, targets, N, B, m, b, p.share, static_cast<float2*>(ws), out, lse};
    hipError_t e;
    if (m == 4) e = go_loss_q<4, CT>(p, a, st);
    else if (m == 8) e = go_loss_q<8, CT>(p, a, st);
    else if (m == 16) e = go_loss_q<16, CT>(p, a, st);
    else if (m == 2 && sizeof(CT) == 1) e = go_loss_q<2, uint8_t>(p, a, st);
    else if (m == 32 && sizeof(CT) == 1) e = go_loss_q<32, uint8_t>(p, a, st);
    else if (m == 64 && sizeof(CT) == 1) e = go_loss_q<64, uint8_t>(p, a, st);
    else e = go_loss_q<0, CT>(p, a, st);
    if (e == hipSuccess && p.shares > 1) {
        hipLaunchKernelGGL(cross_entropy_join_kernel, dim3(B), dim3(kWave), 0, st, a, p.shares, (int)sizeof(CT));
        e = hipGetLastError();
    }
    return record_hip_error(e);
}

template <typename CT>
int backward(const CT* codes, const float* S, const int* targets, const float* lse, const float* grad, long long N, int B, int m, int b,
             float* dS, void* ws, size_t ws_bytes, void* stream) {
    if (!codes || !S || !targets || !lse || !grad || !dS || !ws) return PQ_ERR_NULL;
    int rc = check_shape(N, B, m, b, sizeof(CT));
    if (rc != PQ_OK) return rc;
    Plan p;
    if (!plan_backward(p, N, B, m, b, sizeof(CT))) return PQ_ERR_UNSUPPORTED;
    if (((uintptr_t)codes & 15) || ((uintptr_t)ws & 15) ||
        (((uintptr_t)S | (uintptr_t)targets | (uintptr_t)lse | (uintptr_t)grad | (uintptr_t)dS) & 3))
        return PQ_ERR_ALIGN;
    if (ws_bytes < backward_workspace(p, B, m, b)) return PQ_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    BackArgs a{codes, S, targets, lse, grad, N, B, m, b, p.kept, p.share, static_cast<uint64_t*>(ws), dS};
    hipError_t e;
    if (m == 4) e = go_backward_q<4, CT>(p, a, st);
    else if (m == 8) e = go_backward_q<8, CT>(p, a, st);
    else if (m == 16) e = go_backward_q<16, CT>(p, a, st);
    else if (m == 2 && sizeof(CT) == 1) e = go_backward_q<2, uint8_t>(p, a, st);
    else if (m == 32 && sizeof(CT) == 1) e = go_backward_q<32, uint8_t>(p, a, st);
    else if (m == 64 && sizeof(CT) == 1) e = go_backward_q<64, uint8_t>(p, a, st);
    else e = go_backward_q<0, CT>(p, a, st);
    if (e == hipSuccess && p.shares > 1) {
        const size_t entries = (size_t)B * m * b;
        if (p.shares > kJoinLeads)
            hipLaunchKernelGGL(cross_entropy_backward_join_kernel<kJoinLeads>, dim3((unsigned)ceil_div(entries, kJoinThreads / kJoinLeads)), dim3(kJoinThreads), 0, st, a, p.shares, (int)sizeof(CT));
        else
            hipLaunchKernelGGL(cross_entropy_backward_join_kernel<1>, dim3((unsigned)ceil_div(entries, kJoinThreads)), dim3(kJoinThreads), 0, st, a, p.shares, (int)sizeof(CT));
        e = hipGetLastError();
    }
    return record_hip_error(e);
}

size_t loss_bytes(long long N, int B, int m, int b, int code_bytes) {
    Plan p;
    return check_shape(N, B, m, b, code_bytes) == PQ_OK && plan_loss(p, N, B, m, b, code_bytes) ? loss_workspace(p, B) : 0;
}
size_t backward_bytes(long long N, int B, int m, int b, int code_bytes) {
    Plan p;
    return check_shape(N, B, m, b, code_bytes) == PQ_OK && plan_backward(p, N, B, m, b, code_bytes) ? backward_workspace(p, B, m, b) : 0;
}

}  // namespace
}  // namespace head
}  // namespace pqk

using namespace pqk::head;

extern "C" {

size_t pq_cross_entropy_workspace_bytes(long long N, int B, int m, int b) { return loss_bytes(N, B, m, b, 1); }
size_t pq_cross_entropy_u16_workspace_bytes(long long N, int B, int m, int b) { return loss_bytes(N, B, m, b, 2); }
size_t pq_cross_entropy_backward_workspace_bytes(long long N, int B, int m, int b) { return backward_bytes(N, B, m, b, 1); }
size_t pq_cross_entropy_u16_backward_workspace_bytes(long long N, int B, int m, int b) { return backward_bytes(N, B, m, b, 2); }

int pq_cross_entropy(const uint8_t* codes, const float* S, const int* targets, long long N, int B, int m, int b, float* out, float* lse,
                     void* workspace, size_t workspace_bytes, void* stream) {
    return loss<uint8_t>(codes, S, targets, N, B, m, b, out, lse, workspace, workspace_bytes, stream);
}
int pq_cross_entropy_u16(const uint16_t* codes, const float* S, const int* targets, long long N, int B, int m, int b, float* out, float* lse,
                         void* workspace, size_t workspace_bytes, void* stream) {
    return loss<uint16_t>(codes, S, targets, N, B, m, b, out, lse, workspace, workspace_bytes, stream);
}
int pq_cross_entropy_backward(const uint8_t* codes, const float* S, const int* targets, const float* lse, const float* grad_loss, long long N,
                              int B, int m, int b, float* dS, void* workspace, size_t workspace_bytes, void* stream) {
    return backward<uint8_t>(codes, S, targets, lse, grad_loss, N, B, m, b, dS, workspace, workspace_bytes, stream);
}
int pq_cross_entropy_u16_backward(const uint16_t* codes, const float* S, const int* targets, const float* lse, const float* grad_loss,
                                  long long N, int B, int m, int b, float* dS, void* workspace, size_t workspace_bytes, void* stream) {
    return backward<uint16_t>(codes, S, targets, lse, grad_loss, N, B, m, b, dS, workspace, workspace_bytes, stream);
}

}  // extern "C"
