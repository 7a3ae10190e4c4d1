// Distillation from a teacher's list by the default scorer's W phi (pq_default_distillation), and its gradients.
//
//   w_k = softmax(u / T)   loss = T^2 sum_k w_k (log w_k - log p_k)   dz_i = g T (p_i - sum_{e: item_e = i} w_e)
//
// The passes over W are the cross entropy's at a temperature (default_cross_entropy.hpp).  The listed items' scores are made once more here,
// B K rows of W in 64 bits, for the loss and for the dz of these items, which the gradient's kernels take as it is.
#include "pqtopk_probs.h"
#include "default_cross_entropy.hpp"
#include "teacher.hpp"

namespace pqk {
namespace head {
namespace {

constexpr int kListThreads = 512, kListWaves = kListThreads / kWave;
static_assert(PQ_MAX_K <= kMostEntries && Teacher<kListThreads>::kEach == 1, "a thread an entry");

struct ListArgs {
    const void *W, *H;
    const int* items;
    const float* scores;
    long long N;
    int B, d, K;
    float temperature;
    const float2* partial;     // loss: [groups][B]
    int groups;
    float *loss, *lse;
    const float *lse_in, *grad;                        // gradient
    float* share;
    int* entry_items;
    float* entry_values;
    int few_items, few_groups;                         // default_few_kernel's tiles and workgroups, where it makes the gradient
};

// The list's items' scores in score[].
template <typename T>
__device__ __forceinline__ void score_list(const ListArgs& a, int q, const int* item, double* score) {
    score_rows<kListThreads>(static_cast<const T*>(a.W), static_cast<const T*>(a.H) + (size_t)q * a.d, a.d, a.K, [&](int k) { return (long long)item[k]; },
                             [&](int k, bool there, double z) { if (there) score[k] = z; });
}

// grid = positions: joins the groups' sums, scores the list, adds the loss up.  64 positions with 100 entries 13 us, 1024 with 32 23: rows from memory.
template <typename T>
__global__ __launch_bounds__(kListThreads) void default_distillation_join_kernel(ListArgs a) {
    __shared__ double part[kListWaves], score[kMostEntries];
    __shared__ float2 sums[kListWaves];
    __shared__ int item[kMostEntries];
    const int q = blockIdx.x, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    float c = kLowest, s = 0.0f;
    for (int i = tid; i < a.groups; i += kListThreads) {
        const float2 t = a.partial[(size_t)i * a.B + q];
        join_sums(c, s, t.x, t.y);
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) join_sums(c, s, __shfl_xor(c, x), __shfl_xor(s, x));
    if (lane == 0) sums[wave] = make_float2(c, s);
    const Teacher<kListThreads> t = teacher_of<kListThreads>(a.items, a.scores, q, a.K, a.N, a.temperature, part);
    if (tid < a.K) item[tid] = t.weight[0] != 0.0 ? t.item[0] : -1;       // (of the others no score is asked; NaN is not 0)
    __syncthreads();
    score_list<T>(a, q, item, score);
    __syncthreads();
    c = sums[0].x; s = sums[0].y;
#pragma unroll
    for (int w = 1; w < kListWaves; ++w) join_sums(c, s, sums[w].x, sums[w].y);
    const double lse = log_sum64(c, s);
    const bool live = t.any && lse != -__builtin_inf();
    double loss = live && tid < a.K && item[tid] >= 0 ? entry_loss(t.weight[0], t.log_weight[0], score[tid], a.temperature, lse) : 0.0;
    loss = over_workgroup<kListThreads>(loss, part, [](double x, double y) { return x + y; });
    if (tid == 0) {
        a.lse[q] = (float)lse;
        a.loss[q] = (float)(loss * (double)a.temperature * (double)a.temperature);
    }
}

// grid = positions: the position's share of the gradient and its list in the order of the items (of default_few_kernel's workgroups first), each with p less what the teacher gives the
// item (all its entries together, in the list's order: the same in each of them).  64 positions with 100 entries 16 us, 1024 with 32 15.
template <typename T>
__global__ __launch_bounds__(kListThreads) void default_list_kernel(ListArgs a) {
    __shared__ double part[kListWaves], score[kMostEntries], weight[kMostEntries];
    __shared__ int item[kMostEntries];
    __shared__ long long order[kMostEntries];
    const int q = blockIdx.x, tid = threadIdx.x;
    const Teacher<kListThreads> t = teacher_of<kListThreads>(a.items, a.scores, q, a.K, a.N, a.temperature, part);
    const float lse = a.lse_in[q];
    const bool live = t.any && lse != -__builtin_inff() && a.grad[q] != 0.0f;
    if (tid < a.K) {
        item[tid] = live ? t.item[0] : -1;
        weight[tid] = t.weight[0];
    }
    if (tid == 0) a.share[q] = live ? a.grad[q] * a.temperature : 0.0f;
    __syncthreads();
    score_list<T>(a, q, item, score);
    __syncthreads();
    const int mine = tid >= a.K || item[tid] < 0 ? kNoItem : item[tid];
    // (what orders the entries: the workgroup over the item)
    auto order_of = [&](int i) { return (long long)(a.few_groups ? few_owner(i, a.few_items, a.few_groups) : 0) << 32 | i; };
    if (tid < a.K) order[tid] = order_of(mine);
    __syncthreads();
    if (tid >= a.K) return;
    const long long own = order[tid];
    int rank = 0, alike = 0;
#pragma unroll 8                                               // (reads of LDS on their way together, and no branch between them)
    for (int k = 0; k < a.K; ++k) {
        const long long other = order[k];
        rank += (other < own) | ((other == own) & (k < tid));
        alike += other == own;
    }
    double all = weight[tid];
    if (alike > 1 && mine != kNoItem) {
        all = 0.0;
#pragma unroll 8
        for (int k = 0; k < a.K; ++k) {
            const double w = weight[k];
            all += order[k] == own ? w : 0.0;
        }
    }
    const size_t at = (size_t)q * a.K + rank;
    a.entry_items[at] = mine;
    a.entry_values[at] = mine == kNoItem ? 0.0f : (float)(exp(score[tid] / (double)a.temperature - (double)lse) - all);
}

// What the gradient's workspace holds besides.
struct EntryLayout { size_t share_at, items_at, values_at, bytes; };
EntryLayout lists_of(const DensePlan& p, int B, int K) {
    EntryLayout l;
    l.share_at = round_up(p.bytes, 256);
    l.items_at = round_up(l.share_at + (size_t)B * sizeof(float), 256);
    l.values_at = round_up(l.items_at + (size_t)B * K * sizeof(int), 256);
    l.bytes = round_up(l.values_at + (size_t)B * K * sizeof(float), 256);
    return l;
}

size_t sums_bytes(const DensePlan& p, int B) { return round_up((size_t)p.groups * B * sizeof(float2), 16); }

int check(long long N, int B, int d, int type, int K) {
    if (K < 1) return PQ_ERR_SHAPE;
    const int rc = check_dense(N, B, d, type);
    return rc != PQ_OK ? rc : K > PQ_MAX_K ? PQ_ERR_UNSUPPORTED : PQ_OK;
}

template <typename T>
hipError_t forward(const DensePlan& p, const DenseArgs& a, const ListArgs& l, hipStream_t st) {
    const hipError_t e = dense_loss<T>(p, a, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((default_distillation_join_kernel<T>), dim3(a.B), dim3(kListThreads), 0, st, l);
    return hipGetLastError();
}
template <typename T>
hipError_t backward(const DensePlan& p, const DenseArgs& a, const ListArgs& l, hipStream_t st) {
    hipLaunchKernelGGL((default_list_kernel<T>), dim3(a.B), dim3(kListThreads), 0, st, l);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : dense_backward<T>(p, a, st);
}

}  // namespace
}  // namespace head
}  // namespace pqk

using namespace pqk::head;

extern "C" {

size_t pq_default_distillation_workspace_bytes(long long N, int B, int d, int type, int K) {
    return check(N, B, d, type, K) == PQ_OK ? sums_bytes(plan_dense(N, B, d, type), B) : 0;
}

int pq_default_distillation(const void* W, const void* queries, const int* teacher_items, const float* teacher_scores, long long N, int B, int d, int type,
                            int K, float temperature, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!W || !queries || !teacher_items || !teacher_scores || !loss || !lse || !workspace) return PQ_ERR_NULL;
    if (!(temperature > 0.0f)) return PQ_ERR_SHAPE;
    const int rc = check(N, B, d, type, K);
    if (rc != PQ_OK) return rc;
    if (!temperature_fits(temperature)) return PQ_ERR_UNSUPPORTED;
    if ((((uintptr_t)W | (uintptr_t)queries | (uintptr_t)workspace) & 15) ||
        (((uintptr_t)teacher_items | (uintptr_t)teacher_scores | (uintptr_t)loss | (uintptr_t)lse) & 3))
        return PQ_ERR_ALIGN;
    const DensePlan p = plan_dense(N, B, d, type);
    if (workspace_bytes < sums_bytes(p, B)) return PQ_ERR_WORKSPACE;
    DenseArgs a{};
    a.W = W; a.H = queries; a.N = N; a.B = B; a.d = d; a.scale = (float)(kLog2eDouble / temperature);
    a.item_tiles = p.item_tiles; a.tiles_each = p.tiles_each; a.groups = p.groups; a.position_tiles = p.position_tiles;
    a.partial = static_cast<float2*>(workspace);
    const ListArgs l{W, queries, teacher_items, teacher_scores, N, B, d, K, temperature, a.partial, p.groups, loss, lse, nullptr, nullptr, nullptr, nullptr, nullptr, 0, 0};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return pqk::record_hip_error(type == PQ_FLOAT32 ? forward<float>(p, a, l, st) : type == PQ_BFLOAT16 ? forward<__bf16>(p, a, l, st) : forward<_Float16>(p, a, l, st));
}

size_t pq_default_distillation_backward_workspace_bytes(long long N, int B, int d, int type, int K) {
    return check(N, B, d, type, K) == PQ_OK ? lists_of(plan_dense(N, B, d, type), B, K).bytes : 0;
}

int pq_default_distillation_backward(const void* W, const void* queries, const int* teacher_items, const float* teacher_scores, const float* lse,
                                     const float* grad_loss, long long N, int B, int d, int type, int K, float temperature, void* dqueries, void* dW,
                                     void* workspace, size_t workspace_bytes, void* stream) {
    if (!W || !queries || !teacher_items || !teacher_scores || !lse || !grad_loss || !dqueries || !dW || !workspace) return PQ_ERR_NULL;
    if (!(temperature > 0.0f)) return PQ_ERR_SHAPE;
    const int rc = check(N, B, d, type, K);
    if (rc != PQ_OK) return rc;
    if (!temperature_fits(temperature)) return PQ_ERR_UNSUPPORTED;
    if ((((uintptr_t)W | (uintptr_t)queries | (uintptr_t)workspace | (uintptr_t)dqueries | (uintptr_t)dW) & 15) ||
        (((uintptr_t)teacher_items | (uintptr_t)teacher_scores | (uintptr_t)lse | (uintptr_t)grad_loss) & 3))
        return PQ_ERR_ALIGN;
    const DensePlan p = plan_dense(N, B, d, type);
    const EntryLayout at = lists_of(p, B, K);
    if (workspace_bytes < at.bytes) return PQ_ERR_WORKSPACE;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    DenseArgs a{};
    a.W = W; a.H = queries; a.N = N; a.B = B; a.d = d; a.scale = (float)(kLog2eDouble / temperature);
    a.lse_in = lse; a.grad = grad_loss; a.dH = dqueries; a.dW = dW;
    set_gradient(a, p, workspace);
    float* share = reinterpret_cast<float*>(ws + at.share_at);
    int* entry_items = reinterpret_cast<int*>(ws + at.items_at);
    float* entry_values = reinterpret_cast<float*>(ws + at.values_at);
    a.share = share; a.entry_items = entry_items; a.entry_values = entry_values; a.entries = K;
    const ListArgs l{W, queries, teacher_items, teacher_scores, N, B, d, K, temperature, nullptr, 0, nullptr, nullptr, lse, grad_loss, share, entry_items, entry_values, p.few ? few_items(d) : 0, p.few ? p.slices : 0};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return pqk::record_hip_error(type == PQ_FLOAT32 ? backward<float>(p, a, l, st) : type == PQ_BFLOAT16 ? backward<__bf16>(p, a, l, st) : backward<_Float16>(p, a, l, st));
}

}  // extern "C"
