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
static_assert(PQ_MAX_K <= kMostEntries && kMostEntries <= kListThreads && kMostEntries <= 512, "a thread an entry, whose number has nine bits");

struct ListArgs {
    const void *W, *H;
    const int* items;
    const float* scores;
    long long N;
    int B, d, K;
    float temperature;
    double to_nats;            // of log_sum64()
    const float2* partial;     // loss: [groups][B]
    int groups;
    float *loss, *lse;
    const float *lse_in, *grad;                        // gradient
    float* share;
    int* entry_items;
    float* entry_values;
    int few_items, few_groups;                         // default_few_kernel's tiles and workgroups, where it makes the gradient
};

// A list by a workgroup, a thread an entry: its item (-1: none), its weight and the weight's logarithm, and in score[] its score.  The first wave adds the weights up
// while the others score the items; alone() is called by it after that.
struct Entry {
    int item;
    double weight, log_weight;
    bool any;                  // whether an entry of the list has weight, or is a NaN
};
struct ListMemory {
    double x[kMostEntries], score[kMostEntries];               // of an entry over T; of its item
    int item[kMostEntries];
    WaveTeacher teacher;
};
template <typename T, typename Alone>
__device__ __forceinline__ Entry entry_of(const ListArgs& a, int q, ListMemory& mem, Alone alone) {
    const int tid = threadIdx.x;
    const size_t at = (size_t)q * a.K + min(tid, a.K - 1);
    Entry e;
    e.item = a.items[at];
    const float u = a.scores[at];
    if (tid >= a.K || e.item < 0 || e.item >= a.N) e.item = -1;
    double x = e.item >= 0 ? (double)u / (double)a.temperature : -__builtin_inf();
    if (tid < a.K) {
        mem.item[tid] = e.item;
        mem.x[tid] = x;
    }
    __syncthreads();
    if (tid < kWave) {
        const WaveTeacher t = wave_teacher(a.K, [&](int k) { return mem.x[k]; });
        if (tid == 0) mem.teacher = t;
        alone();
    } else {
        score_rows<kWave, kListThreads>(static_cast<const T*>(a.W), static_cast<const T*>(a.H) + (size_t)q * a.d, a.d, a.K, [&](int k) { return (long long)mem.item[k]; },
                                        [&](int k, bool there, double z) { if (there) mem.score[k] = z; });
    }
    __syncthreads();
    const WaveTeacher t = mem.teacher;
    e.any = t.any;
    if (e.item >= 0) x -= t.top;
    e.weight = !t.any ? 0.0 : t.sum < __builtin_inf() ? t.weight(x) : __builtin_nan("");       // (a list with a NaN or +inf: all of it)
    e.log_weight = x - t.log_sum;
    return e;
}

// grid = positions: joins the groups' sums, scores the list, adds the loss up.  Chains of latencies: one position with 10 entries 4.5 us, 64 with 100 10, 1024 with
// 32 19 (rows from memory).
template <typename T>
__global__ __launch_bounds__(kListThreads) void default_distillation_join_kernel(ListArgs a) {
    __shared__ ListMemory mem;
    __shared__ double part[kListWaves], lse_of_all;
    __shared__ float2 sums[kListWaves];
    const int q = blockIdx.x, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    float c = kLowest, s = 0.0f;
    for (int i = tid; i < a.groups; i += kListThreads) {
        const float2 t = a.partial[(size_t)i * a.B + q];
        join_sums(c, s, t.x, t.y);
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) join_sums(c, s, __shfl_xor(c, x), __shfl_xor(s, x));
    if (lane == 0) sums[wave] = make_float2(c, s);
    const Entry e = entry_of<T>(a, q, mem, [&] {
        float2 t = sums[lane % kListWaves];
#pragma unroll
        for (int x = 1; x < kListWaves; x *= 2) join_sums(t.x, t.y, __shfl_xor(t.x, x), __shfl_xor(t.y, x));
        if (lane == 0) {
            lse_of_all = log_sum64(t.x, t.y, a.to_nats);
            a.lse[q] = (float)lse_of_all;
        }
    });
    const double lse = lse_of_all;
    double loss = e.any && lse != -__builtin_inf() && e.item >= 0 ? entry_loss(e.weight, e.log_weight, mem.score[tid], a.temperature, lse) : 0.0;
    loss = over_workgroup<kListThreads>(loss, part, [](double x, double y) { return x + y; });
    if (tid == 0) a.loss[q] = (float)(loss * (double)a.temperature * (double)a.temperature);
}

// grid = positions: the position's share of the gradient and its list in the order of the items (of default_few_kernel's workgroups first), each with p less what the teacher gives the
// item (all its entries together, in the list's order: the same in each of them).  One position with 10 entries 4 us, 64 with 100 11, and 16 where an item is listed
// ten times; 1024 with 32 12.
template <typename T>
__global__ __launch_bounds__(kListThreads) void default_list_kernel(ListArgs a) {
    __shared__ ListMemory mem;
    __shared__ double weight[kMostEntries], total[kMostEntries];
    __shared__ uint64_t order[kMostEntries], sorted[kMostEntries];
    const int q = blockIdx.x, tid = threadIdx.x;
    const float lse = a.lse_in[q], g = a.grad[q];
    const Entry e = entry_of<T>(a, q, mem, [] {});
    const bool live = e.any && lse != -__builtin_inff() && g != 0.0f;
    if (tid == 0) a.share[q] = live ? g * a.temperature : 0.0f;
    const int mine = live && e.item >= 0 ? e.item : kNoItem;
    // what orders the entries: the workgroup over the item over the entry's place
    const uint64_t owner = a.few_groups ? (mine == kNoItem ? 511 : few_owner(mine, a.few_items, a.few_groups)) : 0;
    const uint64_t own = owner << 41 | (uint64_t)mine << 9 | (uint64_t)tid;
    if (tid < a.K) order[tid] = own;
    __syncthreads();
    int rank = 0;
    if (tid < a.K) {
#pragma unroll 8                                               // (reads of LDS on their way together)
        for (int k = 0; k < a.K; ++k) rank += order[k] < own;
        sorted[rank] = own;
        weight[rank] = e.weight;
    }
    __syncthreads();
    // the first entry of an item adds up what the teacher gives it
    if (tid < a.K && (rank == 0 || sorted[rank - 1] >> 9 != own >> 9)) {
        double all = e.weight;
        int end = rank + 1;
        for (bool more = end < a.K; more;) {                   // (four at once: a list may hold an item many times)
            uint64_t key[4];
            double w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                key[i] = sorted[min(end + i, a.K - 1)];
                w[i] = weight[min(end + i, a.K - 1)];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                more = more && end < a.K && key[i] >> 9 == own >> 9;
                all += more ? w[i] : 0.0;
                end += more;
            }
        }
        for (int i = rank; i < end; ++i) total[i] = all;
    }
    __syncthreads();
    if (tid >= a.K) return;
    const size_t at = (size_t)q * a.K + rank;
    a.entry_items[at] = mine;
    a.entry_values[at] = mine == kNoItem ? 0.0f : (float)(exp(mem.score[tid] / (double)a.temperature - (double)lse) - total[rank]);
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
hipError_t forward(const DensePlan& p, const DenseLossArgs& a, const ListArgs& l, hipStream_t st) {
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
    DenseLossArgs a{};
    a.W = W; a.H = queries; a.N = N; a.B = B; a.d = d; a.scale = (float)(kLog2eDouble / temperature);
    a.item_tiles = p.item_tiles; a.tiles_each = p.tiles_each; a.groups = p.groups; a.position_tiles = p.position_tiles;
    a.partial = static_cast<float2*>(workspace);
    const ListArgs l{W, queries, teacher_items, teacher_scores, N, B, d, K, temperature, 1.0 / base_of(a.scale, temperature), a.partial, p.groups, loss, lse, nullptr, nullptr, nullptr, nullptr, nullptr, 0, 0};
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
    a.base = base_of(a.scale, temperature);
    a.lse_in = lse; a.grad = grad_loss; a.dH = dqueries; a.dW = dW;
    set_gradient(a, p, workspace);
    float* share = reinterpret_cast<float*>(ws + at.share_at);
    int* entry_items = reinterpret_cast<int*>(ws + at.items_at);
    float* entry_values = reinterpret_cast<float*>(ws + at.values_at);
    a.share = share; a.entry_items = entry_items; a.entry_values = entry_values; a.entries = K;
    const ListArgs l{W, queries, teacher_items, teacher_scores, N, B, d, K, temperature, 0.0, nullptr, 0, nullptr, nullptr, lse, grad_loss, share, entry_items, entry_values, p.few ? few_items(d) : 0, p.few ? p.slices : 0};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return pqk::record_hip_error(type == PQ_FLOAT32 ? backward<float>(p, a, l, st) : type == PQ_BFLOAT16 ? backward<__bf16>(p, a, l, st) : backward<_Float16>(p, a, l, st));
}

}  // extern "C"
