// Log-probabilities of given items, entropy and the likeliest items by sub-ids (pq_log_probs*): one pass over the codebook whose lookups
// serve all of them.
//
//   r_qi = sum_k S[q][k][G[i][k]]   lse = log sum_i exp(r_i / T)   log p_i = r_i / T - lse   entropy = lse - sum_i p_i r_i / T
//
// The pass is the cross entropy's (cross_entropy.hpp) with one more sum.  The likeliest items come from it too, what scores pass a position's floor going to
// its list (alternatives.hpp), or, where the lookups are few, from the ranking's own scan, whose bounds of one byte need no first piece and no cut (by_ranking()).
// Bound by the vector units, with the lookups in LDS close behind: 64 positions of 1.27M items, m = 8, one and a half times the loss's vector instructions, whose issue takes all of the time
// (80 % of the loss's), LDS busy 84 % of it (89 %).  512 positions, K = 100, 517 to 553 us; two launches of 6.8 and 5.7 us for one position of 10,000.
#include "pqtopk_probs.h"
#include "cross_entropy.hpp"

namespace pqk {
namespace head {
namespace subids {
namespace {

// Two workgroups a compute unit, 64 registers a lane, but for rows of 16 and 32 bytes (as the loss has it, see plan_loss()).
template <int M, typename CT, int Q>
__global__ __launch_bounds__(kThreads, (waves_of<M, CT, ProbsArgs>())) void log_probs_kernel(ProbsArgs a) { sum_items<M, CT, Q, true>(a); }

struct FinishArgs {
    const void* codes;
    const float* S;
    const int* items;
    long long N;
    int B, m, b, n, K, code_bytes;
    double per_temperature, to_nats;                   // 1 / T; of log_sum64()
    const float4* partial;     // [B][shares]
    int shares, stored, regions;                       // shares of all pieces; of the last piece what cut_list() takes
    long long region;
    Lists lists;
    const float* ranked;       // [B][K], or NULL: the scores of top_items, which a ranking has found
    float *log_probs, *entropy, *lse;
    int* top_items;
    float* top_log_probs;
};

// Eq. 5's chain of one item, from the tables where they lie; -inf where a sub-id is out of play.
__device__ __forceinline__ float score_of_item(const FinishArgs& a, int q, int item) {
    float z = 0.0f;
#pragma unroll 8                                               // (a chain of additions, but not of loads)
    for (int k = 0; k < a.m; ++k) {
        const size_t at = (size_t)item * a.m + k;
        const uint32_t g = a.code_bytes == 1 ? (uint32_t)static_cast<const uint8_t*>(a.codes)[at] : (uint32_t)static_cast<const uint16_t*>(a.codes)[at];
        float v = a.S[((size_t)q * a.m + k) * a.b + min(g, (uint32_t)a.b - 1u)];
        v = v < kLeastEntry ? kLeastEntry : v;
        z = k == 0 ? v : z + v;
    }
    return z < kNoScore ? -__builtin_inff() : z + 0.0f;
}

// grid = positions: joins the shares' sums, scores the given items, cuts the list to the K best and puts them in order.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void log_probs_finish_kernel(FinishArgs a) {
    __shared__ SelectMemory<THREADS> mem;
    __shared__ uint64_t kept[kMostKept];
    __shared__ float4 sums[THREADS / kWave];
    __shared__ double lse_of_all;
    constexpr int kWaves = THREADS / kWave;
    const int q = blockIdx.x, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    // the given item that a thread scores aside, in a wave that has no other work there: what its row takes to come is over by then
    const int own = (tid + THREADS / 2) % THREADS;
    int item = own < a.n ? a.items[(size_t)q * a.n + own] : -1;
    uint8_t touched = 0;
    float given = 0.0f;
    auto own_sums = [&] {
        float c = kLowest, s = 0.0f, t = 0.0f;
        for (int i = tid; i < a.shares; i += THREADS) {
            const float4 v = a.partial[(size_t)q * a.shares + i];
            join_sums(c, s, t, v.x, v.y, v.z);
        }
        if (wave * kWave < a.shares) join_wave(c, s, t);
        if (lane == 0) sums[wave] = make_float4(c, s, t, 0.0f);
        item = item < a.N ? item : -1;
        if (item >= 0) touched = static_cast<const uint8_t*>(a.codes)[(size_t)item * a.m * a.code_bytes];
    };
    auto aside = [&] {
        asm volatile("" ::"v"((int)touched));
        if (item >= 0) given = score_of_item(a, q, item);
        if (wave != kWaves - 1) return;
        float4 v = sums[lane % kWaves];                        // (64-bit logarithms, by one wave)
        join_wave<kWaves>(v.x, v.y, v.z);
        if (lane == 0) {
            lse_of_all = log_sum64(v.x, v.y, a.to_nats);
            a.lse[q] = (float)lse_of_all;
            a.entropy[q] = entropy_of(v.y, v.z);
        }
    };
    uint64_t least;
    bool sorted = false;
    int n = 0;
    if (a.lists.keep) n = cut_list<THREADS>(a.lists, q, a.stored, a.regions, a.region, true, kept, sorted, least, mem, own_sums, aside);
    else {
        own_sums();
        __syncthreads();
        aside();
        __syncthreads();
    }
    const double lse = lse_of_all;
    auto log_prob = [&](float z) { return log_prob_of((double)z * a.per_temperature, lse); };
    if (own < a.n) a.log_probs[(size_t)q * a.n + own] = item >= 0 ? log_prob(given) : 0.0f;
    for (int i = own + THREADS; i < a.n; i += THREADS) {
        const int next = a.items[(size_t)q * a.n + i];
        a.log_probs[(size_t)q * a.n + i] = next >= 0 && next < a.N ? log_prob(score_of_item(a, q, next)) : 0.0f;
    }
    if (a.K == 0) return;
    if (a.ranked) {
        // (the ranking took scores of -inf for sums of large numbers: fewer than K others mean that K - 1 ids hold enough of them, the lowest ones)
        __shared__ int below[PQ_MAX_K];
        if (lse != lse) {                                      // (its ids are some items)
            for (int i = tid; i < a.K; i += THREADS) a.top_log_probs[(size_t)q * a.K + i] = (float)lse;
            return;
        }
        const float last = a.ranked[(size_t)q * a.K + a.K - 1];
        for (int i = tid; i < a.K; i += THREADS) {
            const float z = a.ranked[(size_t)q * a.K + i];
            if (z >= kNoScore) a.top_log_probs[(size_t)q * a.K + i] = log_prob(z);
            if (last < kNoScore) below[i] = score_of_item(a, q, i) < kNoScore;
        }
        __syncthreads();
        if (last >= kNoScore) return;
        int others = 0;
        for (int i = 0; i < a.K; ++i) others += a.ranked[(size_t)q * a.K + i] >= kNoScore;
        for (int i = tid; i < a.K; i += THREADS) {
            int rank = others;
            for (int j = 0; j < i; ++j) rank += below[j];
            if (below[i] && rank < a.K) {
                a.top_items[(size_t)q * a.K + rank] = i;
                a.top_log_probs[(size_t)q * a.K + rank] = -__builtin_inff();
            }
        }
        return;
    }
    for (int at = tid; at < n; at += THREADS) {
        const uint64_t mine = kept[at];
        int rank = sorted ? at : 0;
        if (!sorted) {
#pragma unroll 8                                               // (their reads of LDS on their way together)
            for (int i = 0; i < n; ++i) rank += kept[i] > mine;
        }
        if (rank < a.K) {
            a.top_items[(size_t)q * a.K + rank] = (int)item_of(mine);
            a.top_log_probs[(size_t)q * a.K + rank] = log_prob(score_of(mine));
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------
// host side

template <int M, typename CT, int Q>
hipError_t go(const Plan& p, const ProbsArgs& a, hipStream_t st) {
    hipError_t e = allow_lds(log_probs_kernel<M, CT, Q>, p.lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((log_probs_kernel<M, CT, Q>), dim3(p.shares, p.groups), dim3(kThreads), p.lds, st, a);
    return hipGetLastError();
}
template <int M, typename CT>
hipError_t go_q(const Plan& p, const ProbsArgs& a, hipStream_t st) {
    if constexpr (fits<M, CT>(4, 0)) { if (p.Q == 4) return go<M, CT, 4>(p, a, st); }
    if (p.Q == 2) return go<M, CT, 2>(p, a, st);
    return go<M, CT, 1>(p, a, st);
}
template <typename CT>
hipError_t go_m(const Plan& p, const ProbsArgs& a, hipStream_t st) {
    if (a.m == 4) return go_q<4, CT>(p, a, st);
    if (a.m == 8) return go_q<8, CT>(p, a, st);
    if (a.m == 16) return go_q<16, CT>(p, a, st);
    if (a.m == 2 && sizeof(CT) == 1) return go_q<2, uint8_t>(p, a, st);
    if (a.m == 32 && sizeof(CT) == 1) return go_q<32, uint8_t>(p, a, st);
    if (a.m == 64 && sizeof(CT) == 1) return go_q<64, uint8_t>(p, a, st);
    return go_q<0, CT>(p, a, st);
}

// Where the workspace's parts lie.
struct Layout : ListLayout {
    Passes passes;
    Sums sums;
    size_t topk_bytes, finite_at, ranked_at, topk_at;          // (topk_bytes: 0 where lists are kept)
};
// Whether the ranking's scan follows the pass instead of lists.  It looks the items up again, in chains that grow with m; lists take launches, more of them for a larger K, and cuts
// of up to kFewKept keys take less.  All of a call, us, lists and scan, K = 10 and 100: 1.28M items, m = 8: 4 positions 42 | 39, 57 | 44; 16 50 | 55, 65 | 60; 64 94 | 105,
// 113 | 118; m = 16: 4 55 | 50, 68 | 56; 16 70 | 74, 84 | 81; 64 147 | 178, 165 | 195; m = 4: 16 45 | 44, 62 | 48; 64 77 | 79, 102 | 86; 400,000 items, m = 32: 4 58 | 56,
// 66 | 60; 16 58 | 82, 66 | 89; 200,000, m = 8: 32 42 | 39, 51 | 47; 64 46 | 49, 56 | 55; 5M, m = 8: 4 57 | 56, 149 | 61; 16 97 | 105, 186 | 112; 64 270 | 292, 301 | 330;
// 50,000, m = 8: 200 47 | 46, 55 | 55; 400 58 | 63, 71 | 97; 1000 82 | 102, 102 | 142; 300,000, m = 4: 400 122 | 107, 137 | 125.
// Two of these points lie on the rule's slower side: the last one (m^2 makes too much of four splits), by 14 and 10 %, and 1.28M, m = 8, 64 positions, K = 100, by 4 %.  All are of one-byte
// sub-ids; those of two bytes follow the same rule unmeasured.
bool by_ranking(long long N, int B, int m, int K) { return K > 0 && N > kOnePiece && (double)N * B * m * m <= (K <= kFewKept || B >= 128 ? 1.2e9 : 6e9); }
size_t topk_bytes_of(long long N, int B, int m, int b, int K, int code_bytes) {
    if (!by_ranking(N, B, m, K)) return 0;
    return code_bytes == 1 ? pq_score_topk_workspace_bytes(N, B, m, b, K) : pq_score_topk_u16_workspace_bytes(N, B, m, b, K);
}
bool lay_out(Layout& l, long long N, int B, int m, int b, int K, int code_bytes) {
    l.topk_bytes = topk_bytes_of(N, B, m, b, K, code_bytes);
    l.passes = passes_of(N, B, l.topk_bytes ? 0 : K);
    l.sums = Sums();
    for (long long done = 0, now; done < N; done += now) {
        Plan p;
        now = l.passes.after(done);
        if (!plan_loss(p, now, B, m, b, code_bytes, kListedBytes)) return false;
        l.sums.piece(p.shares);
        l.piece(done == 0 ? now : (long long)p.shares * p.share);
    }
    l.sums.lay_out(B);
    l.ListLayout::lay_out(l.sums.bytes(B), B, l.passes);
    if (l.topk_bytes) {
        l.finite_at = l.bytes;
        l.ranked_at = l.finite_at + round_up((size_t)B * m * b * sizeof(float), 256);
        l.topk_at = l.ranked_at + round_up((size_t)B * K * sizeof(float), 256);
        l.bytes = l.topk_at + round_up(l.topk_bytes, 256);
    }
    return true;
}

int check(long long N, int B, int m, int b, int K, int code_bytes) {
    if (K < 0 || K > N) return PQ_ERR_SHAPE;
    const int rc = check_shape(N, B, m, b, code_bytes);
    return rc != PQ_OK ? rc : K > PQ_MAX_K ? PQ_ERR_UNSUPPORTED : PQ_OK;
}

size_t bytes_of(long long N, int B, int m, int b, int K, int code_bytes) {
    Layout l;
    return check(N, B, m, b, K, code_bytes) == PQ_OK && lay_out(l, N, B, m, b, K, code_bytes) ? l.bytes : 0;
}

template <typename CT>
int log_probs(const CT* codes, const float* S, const int* items, long long N, int B, int m, int b, int n, int K, float temperature, float* out,
              float* entropy, float* lse, int* top_items, float* top_log_probs, void* workspace, size_t ws_bytes, void* stream) {
    if (!codes || !S || !entropy || !lse || !workspace || (n != 0 && (!items || !out)) || (K != 0 && (!top_items || !top_log_probs))) return PQ_ERR_NULL;
    if (n < 0 || !(temperature > 0.0f)) return PQ_ERR_SHAPE;
    int rc = check(N, B, m, b, K, sizeof(CT));
    if (rc != PQ_OK) return rc;
    Layout l;
    if (n > kMostGiven || !temperature_fits(temperature) || !lay_out(l, N, B, m, b, K, sizeof(CT))) return PQ_ERR_UNSUPPORTED;
    if ((((uintptr_t)codes | (uintptr_t)workspace) & 15) || (((uintptr_t)S | (uintptr_t)entropy | (uintptr_t)lse) & 3) ||
        (n && (((uintptr_t)items | (uintptr_t)out) & 3)) || (K && (((uintptr_t)top_items | (uintptr_t)top_log_probs) & 3)))
        return PQ_ERR_ALIGN;
    if (ws_bytes < l.bytes) return PQ_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    const Lists lists = l.lists(ws, l.passes.keep);
    ProbsArgs a{codes, S, N, B, m, b, 0, (float)(kLog2eDouble / temperature), 0, 0, 0, reinterpret_cast<float4*>(ws), l.sums.slots, 0, 0, lists,
                l.topk_bytes ? reinterpret_cast<float*>(ws + l.finite_at) : nullptr};
    float* ranked = l.topk_bytes ? reinterpret_cast<float*>(ws + l.ranked_at) : nullptr;
    hipError_t e = hipSuccess;
    Plan p;
    for (long long done = 0; done < N && e == hipSuccess; done = a.end) {
        const long long now = l.passes.after(done);
        plan_loss(p, now, B, m, b, sizeof(CT), kListedBytes);
        a.first = (uint32_t)done;
        a.end = (uint32_t)(done + now);
        a.share = p.share;
        a.store = lists.keep != 0 && done == 0;
        e = go_m<CT>(p, a, st);
        l.sums.advance(p.shares, a.done, a.written);
        if (e == hipSuccess && lists.keep && a.end < N) e = launch_select(lists, B, a.store ? (int)now : 0, p.shares, p.share, st);
    }
    if (e == hipSuccess && ranked) {
        if (sizeof(CT) == 1) rc = pq_score_topk(reinterpret_cast<const uint8_t*>(codes), a.finite, N, B, m, b, K, top_items, ranked, ws + l.topk_at, l.topk_bytes, stream);
        else rc = pq_score_topk_u16(reinterpret_cast<const uint16_t*>(codes), a.finite, N, B, m, b, K, top_items, ranked, ws + l.topk_at, l.topk_bytes, stream);
        if (rc != PQ_OK) return rc;
    }
    if (e == hipSuccess) {
        const FinishArgs f{codes, S, items, N, B, m, b, n, K, (int)sizeof(CT), 1.0 / temperature, 1.0 / base_of(a.scale, temperature), reinterpret_cast<const float4*>(ws), l.sums.slots,
                           a.store ? (int)N : 0, p.shares, p.share, lists, ranked, out, entropy, lse, top_items, top_log_probs};
        if (many_lists(B) || lists.keep == 0) hipLaunchKernelGGL(log_probs_finish_kernel<256>, dim3(B), dim3(256), 0, st, f);
        else hipLaunchKernelGGL(log_probs_finish_kernel<1024>, dim3(B), dim3(1024), 0, st, f);
        e = hipGetLastError();
    }
    return record_hip_error(e);
}

}  // namespace
}  // namespace subids
}  // namespace head
}  // namespace pqk

using namespace pqk::head::subids;

extern "C" {

size_t pq_log_probs_workspace_bytes(long long N, int B, int m, int b, int K) { return bytes_of(N, B, m, b, K, 1); }
size_t pq_log_probs_u16_workspace_bytes(long long N, int B, int m, int b, int K) { return bytes_of(N, B, m, b, K, 2); }

int pq_log_probs(const uint8_t* codes, const float* S, const int* items, long long N, int B, int m, int b, int n, int K, float temperature,
                 float* out, float* entropy, float* lse, int* top_items, float* top_log_probs, void* workspace, size_t workspace_bytes, void* stream) {
    return log_probs<uint8_t>(codes, S, items, N, B, m, b, n, K, temperature, out, entropy, lse, top_items, top_log_probs, workspace, workspace_bytes, stream);
}
int pq_log_probs_u16(const uint16_t* codes, const float* S, const int* items, long long N, int B, int m, int b, int n, int K, float temperature,
                     float* out, float* entropy, float* lse, int* top_items, float* top_log_probs, void* workspace, size_t workspace_bytes, void* stream) {
    return log_probs<uint16_t>(codes, S, items, N, B, m, b, n, K, temperature, out, entropy, lse, top_items, top_log_probs, workspace, workspace_bytes, stream);
}

}  // extern "C"
