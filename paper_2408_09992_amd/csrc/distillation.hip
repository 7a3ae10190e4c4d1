// Distillation from a teacher's list by sub-ids (pq_distillation*): the softmax of the whole catalogue against a few items' weights.
//
//   w_k = softmax(u / T)   loss = T^2 sum_k w_k (log w_k - log p_k)   dS[k][j] = g T (sum_{i: G[i][k] = j} p_i - sum_{e: G[item_e][k] = j} w_e)
//
// Both passes over the codebook are the cross entropy's at a temperature (cross_entropy.hpp).  The teacher's weights, whole multiples of
// 2^-62 as the probabilities are, are one more share of the gradient's sums, with the sign turned: they meet in the join.
#include "pqtopk_probs.h"
#include "cross_entropy.hpp"
#include "teacher.hpp"

namespace pqk {
namespace head {
namespace subids {
namespace {

constexpr int kTeacherThreads = 256, kTeacherWaves = kTeacherThreads / kWave, kEach = Teacher<kTeacherThreads>::kEach;

struct TeacherArgs {
    const void* codes;
    const float* S;
    const int* items;
    const float* scores;
    long long N;
    int B, m, b, K, code_bytes;
    float temperature;
    const float2* partial;     // loss: [shares][B]
    int shares;
    float *loss, *lse;
    const float *lse_in, *grad;
    uint64_t* mass;            // gradient: [B][m][b]
    float* weight;             // [B]
};

__device__ __forceinline__ uint32_t code_of(const TeacherArgs& a, int item, int k) {
    const size_t at = (size_t)item * a.m + k;
    const uint32_t g = a.code_bytes == 1 ? (uint32_t)static_cast<const uint8_t*>(a.codes)[at] : (uint32_t)static_cast<const uint16_t*>(a.codes)[at];
    return min(g, (uint32_t)a.b - 1u);
}

// grid = positions: joins the shares' sums and scores the list's items, Eq. 5's chain each.
__global__ __launch_bounds__(kTeacherThreads) void distillation_join_kernel(TeacherArgs a) {
    __shared__ double part[kTeacherWaves];
    __shared__ float2 sums[kTeacherWaves];
    const int q = blockIdx.x, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    float c = kLowest, s = 0.0f;
    for (int i = tid; i < a.shares; i += kTeacherThreads) {
        const float2 t = a.partial[(size_t)i * a.B + q];
        join_sums(c, s, t.x, t.y);
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) join_sums(c, s, __shfl_xor(c, x), __shfl_xor(s, x));
    if (lane == 0) sums[wave] = make_float2(c, s);
    const Teacher<kTeacherThreads> t = teacher_of<kTeacherThreads>(a.items, a.scores, q, a.K, a.N, a.temperature, part);
    c = sums[0].x; s = sums[0].y;
#pragma unroll
    for (int w = 1; w < kTeacherWaves; ++w) join_sums(c, s, sums[w].x, sums[w].y);
    const float lse = log_sum(c, s);
    const bool live = t.any && lse != -__builtin_inff();
    const double lse64 = lse == lse ? ((double)c + log2((double)s)) / kLog2eDouble : (double)lse;
    double loss = 0.0;
    if (live) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (t.item[j] < 0) continue;
            float z = 0.0f;
            for (int k = 0; k < a.m; ++k) {
                const float v = a.S[((size_t)q * a.m + k) * a.b + code_of(a, t.item[j], k)];
                z = k == 0 ? v : z + v;
            }
            loss += entry_loss(t.weight[j], t.log_weight[j], z, a.temperature, lse64);
        }
    }
    loss = over_workgroup<kTeacherThreads>(loss, part, [](double x, double y) { return x + y; });
    if (tid == 0) {
        a.lse[q] = lse;
        a.loss[q] = (float)(loss * (double)a.temperature * (double)a.temperature);
    }
}

// grid = positions: what the gradient's kernels need of a position, and the share of the sums that is the teacher's.
constexpr int kMassEntries = 8192;                     // of a table at once (64 KB of LDS)
__global__ __launch_bounds__(kTeacherThreads) void teacher_mass_kernel(TeacherArgs a) {
    __shared__ double part[kTeacherWaves];
    __shared__ unsigned long long mass[kMassEntries];
    const int q = blockIdx.x, tid = threadIdx.x, entries = a.m * a.b;
    const Teacher<kTeacherThreads> t = teacher_of<kTeacherThreads>(a.items, a.scores, q, a.K, a.N, a.temperature, part);
    const bool live = t.any && a.lse_in[q] != -__builtin_inff();
    if (tid == 0) a.weight[q] = !live ? 0.0f : t.odd ? __builtin_nanf("") : a.grad[q] * a.temperature;
    for (int first = 0; first < entries; first += kMassEntries) {
        const int here = min(kMassEntries, entries - first);
        for (int i = tid; i < here; i += kTeacherThreads) mass[i] = 0;
        __syncthreads();
        if (live && !t.odd) {
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                if (t.item[j] < 0) continue;
                const unsigned long long fixed = (unsigned long long)(t.weight[j] * 0x1p62);
                for (int k = 0; k < a.m; ++k) {
                    const int at = k * a.b + (int)code_of(a, t.item[j], k) - first;
                    if (at >= 0 && at < here) atomicAdd(&mass[at], 0ull - fixed);          // (whole numbers: the order changes nothing)
                }
            }
        }
        __syncthreads();
        for (int i = tid; i < here; i += kTeacherThreads) a.mass[(size_t)q * entries + first + i] = mass[i];
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------------
// host side

int check(long long N, int B, int m, int b, int K, int code_bytes) {
    if (K < 1) return PQ_ERR_SHAPE;
    const int rc = check_shape(N, B, m, b, code_bytes);
    return rc != PQ_OK ? rc : K > PQ_MAX_K ? PQ_ERR_UNSUPPORTED : PQ_OK;
}
static_assert(PQ_MAX_K <= kMostEntries, "a list");

size_t sums_bytes(const Plan& p, int B) { return round_up((size_t)p.shares * B * sizeof(float2), 16); }
size_t masses_bytes(const Plan& p, int B, int m, int b) { return round_up((size_t)(p.shares + 1) * B * m * b * sizeof(uint64_t), 256); }

template <typename CT>
int distil(const CT* codes, const float* S, const int* items, const float* scores, long long N, int B, int m, int b, int K, float temperature, float* loss,
           float* lse, void* ws, size_t ws_bytes, void* stream) {
    if (!codes || !S || !items || !scores || !loss || !lse || !ws) return PQ_ERR_NULL;
    if (!(temperature > 0.0f)) return PQ_ERR_SHAPE;
    const int rc = check(N, B, m, b, K, sizeof(CT));
    if (rc != PQ_OK) return rc;
    Plan p;
    if (!temperature_fits(temperature) || !plan_loss(p, N, B, m, b, sizeof(CT))) return PQ_ERR_UNSUPPORTED;
    if ((((uintptr_t)codes | (uintptr_t)ws) & 15) || (((uintptr_t)S | (uintptr_t)items | (uintptr_t)scores | (uintptr_t)loss | (uintptr_t)lse) & 3)) return PQ_ERR_ALIGN;
    if (ws_bytes < sums_bytes(p, B)) return PQ_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const LossArgs a{codes, S, nullptr, N, B, m, b, p.share, static_cast<float2*>(ws), nullptr, nullptr, (float)(kLog2eDouble / temperature)};
    hipError_t e = launch_loss(p, a, sizeof(CT), st);
    if (e == hipSuccess) {
        TeacherArgs t{codes, S, items, scores, N, B, m, b, K, (int)sizeof(CT), temperature, a.partial, p.shares, loss, lse, nullptr, nullptr, nullptr, nullptr};
        hipLaunchKernelGGL(distillation_join_kernel, dim3(B), dim3(kTeacherThreads), 0, st, t);
        e = hipGetLastError();
    }
    return record_hip_error(e);
}

template <typename CT>
int distil_backward(const CT* codes, const float* S, const int* items, const float* scores, const float* lse, const float* grad, long long N, int B, int m,
                    int b, int K, float temperature, float* dS, void* ws, size_t ws_bytes, void* stream) {
    if (!codes || !S || !items || !scores || !lse || !grad || !dS || !ws) return PQ_ERR_NULL;
    if (!(temperature > 0.0f)) return PQ_ERR_SHAPE;
    const int rc = check(N, B, m, b, K, sizeof(CT));
    if (rc != PQ_OK) return rc;
    Plan p;
    if (!temperature_fits(temperature) || !plan_backward(p, N, B, m, b, sizeof(CT))) return PQ_ERR_UNSUPPORTED;
    if ((((uintptr_t)codes | (uintptr_t)ws) & 15) ||
        (((uintptr_t)S | (uintptr_t)items | (uintptr_t)scores | (uintptr_t)lse | (uintptr_t)grad | (uintptr_t)dS) & 3))
        return PQ_ERR_ALIGN;
    const size_t mass_bytes = masses_bytes(p, B, m, b);
    if (ws_bytes < mass_bytes + (size_t)B * sizeof(float)) return PQ_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    uint64_t* partial = static_cast<uint64_t*>(ws);
    float* weight = reinterpret_cast<float*>(static_cast<unsigned char*>(ws) + mass_bytes);
    const TeacherArgs t{codes, S, items, scores, N, B, m, b, K, (int)sizeof(CT), temperature, nullptr, 0, nullptr, nullptr, lse, grad,
                        partial + (size_t)p.shares * B * m * b, weight};
    hipLaunchKernelGGL(teacher_mass_kernel, dim3(B), dim3(kTeacherThreads), 0, st, t);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) {
        const BackArgs a{codes, S, nullptr, lse, grad, N, B, m, b, p.kept, p.share, partial, dS, weight, (float)(kLog2eDouble / temperature)};
        e = launch_backward(p, a, sizeof(CT), p.shares + 1, st);
    }
    return record_hip_error(e);
}

size_t forward_bytes(long long N, int B, int m, int b, int K, int code_bytes) {
    Plan p;
    return check(N, B, m, b, K, code_bytes) == PQ_OK && plan_loss(p, N, B, m, b, code_bytes) ? sums_bytes(p, B) : 0;
}
size_t back_bytes(long long N, int B, int m, int b, int K, int code_bytes) {
    Plan p;
    return check(N, B, m, b, K, code_bytes) == PQ_OK && plan_backward(p, N, B, m, b, code_bytes) ? round_up(masses_bytes(p, B, m, b) + (size_t)B * sizeof(float), 16) : 0;
}

}  // namespace
}  // namespace subids
}  // namespace head
}  // namespace pqk

using namespace pqk::head::subids;

extern "C" {

size_t pq_distillation_workspace_bytes(long long N, int B, int m, int b, int K) { return forward_bytes(N, B, m, b, K, 1); }
size_t pq_distillation_u16_workspace_bytes(long long N, int B, int m, int b, int K) { return forward_bytes(N, B, m, b, K, 2); }
size_t pq_distillation_backward_workspace_bytes(long long N, int B, int m, int b, int K) { return back_bytes(N, B, m, b, K, 1); }
size_t pq_distillation_u16_backward_workspace_bytes(long long N, int B, int m, int b, int K) { return back_bytes(N, B, m, b, K, 2); }

int pq_distillation(const uint8_t* codes, const float* S, const int* teacher_items, const float* teacher_scores, long long N, int B, int m, int b, int K,
                    float temperature, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    return distil<uint8_t>(codes, S, teacher_items, teacher_scores, N, B, m, b, K, temperature, loss, lse, workspace, workspace_bytes, stream);
}
int pq_distillation_u16(const uint16_t* codes, const float* S, const int* teacher_items, const float* teacher_scores, long long N, int B, int m, int b, int K,
                        float temperature, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    return distil<uint16_t>(codes, S, teacher_items, teacher_scores, N, B, m, b, K, temperature, loss, lse, workspace, workspace_bytes, stream);
}
int pq_distillation_backward(const uint8_t* codes, const float* S, const int* teacher_items, const float* teacher_scores, const float* lse,
                             const float* grad_loss, long long N, int B, int m, int b, int K, float temperature, float* dS, void* workspace,
                             size_t workspace_bytes, void* stream) {
    return distil_backward<uint8_t>(codes, S, teacher_items, teacher_scores, lse, grad_loss, N, B, m, b, K, temperature, dS, workspace, workspace_bytes, stream);
}
int pq_distillation_u16_backward(const uint16_t* codes, const float* S, const int* teacher_items, const float* teacher_scores, const float* lse,
                                 const float* grad_loss, long long N, int B, int m, int b, int K, float temperature, float* dS, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    return distil_backward<uint16_t>(codes, S, teacher_items, teacher_scores, lse, grad_loss, N, B, m, b, K, temperature, dS, workspace, workspace_bytes, stream);
}

}  // extern "C"
