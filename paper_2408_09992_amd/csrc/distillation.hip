// Distillation from a teacher's list by sub-ids (pq_distillation*): the softmax of the whole catalogue against a few items' weights.
//
//   w_k = softmax(u / T)   loss = T^2 sum_k w_k (log w_k - log p_k)   dS[k][j] = g T (sum_{i: G[i][k] = j} p_i - sum_{e: G[item_e][k] = j} w_e)
//
// Both passes over the codebook are the cross entropy's at a temperature (cross_entropy.hpp), whose kernels take a list in the place of a target:
// one wave of a workgroup makes its weights and, in the loss, scores its items; the gradient's sums start from what the teacher gives, below 0.
// Bound by LDS as the cross entropy is: 256 positions of 1.27M items, m = 8, lists of 100: loss 209 us, gradient 767; a list adds some 2 us to each where there is one position of 10,000 items.
#include "pqtopk_probs.h"
#include "cross_entropy.hpp"
#include "teacher.hpp"

namespace pqk {
namespace head {
namespace subids {
namespace {

// ---------------------------------------------------------------------------------------------------------------
// host side

int check(long long N, int B, int m, int b, int K, int code_bytes) {
    if (K < 1) return PQ_ERR_SHAPE;
    const int rc = check_shape(N, B, m, b, code_bytes);
    return rc != PQ_OK ? rc : K > PQ_MAX_K ? PQ_ERR_UNSUPPORTED : PQ_OK;
}

size_t masses_bytes(const Plan& p, int B, int m, int b) { return round_up(backward_workspace(p, B, m, b), 256); }

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
    if (ws_bytes < loss_workspace(p, B)) return PQ_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const float scale = (float)(kLog2eDouble / temperature);
    const TeacherLossArgs a{{codes, S, nullptr, N, B, m, b, p.share, static_cast<float2*>(ws), loss, lse, scale}, items, scores, K, temperature, 1.0 / base_of(scale, temperature)};
    return record_hip_error(launch_loss<CT>(p, a, st));
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
    const float scale = (float)(kLog2eDouble / temperature);
    const TeacherBackArgs a{{codes, S, nullptr, lse, grad, N, B, m, b, p.kept, p.share, partial, dS, scale, base_of(scale, temperature)}, items, scores, K, temperature, weight};
    return record_hip_error(launch_backward<CT>(p, a, st));
}

size_t forward_bytes(long long N, int B, int m, int b, int K, int code_bytes) {
    Plan p;
    return check(N, B, m, b, K, code_bytes) == PQ_OK && plan_loss(p, N, B, m, b, code_bytes) ? loss_workspace(p, B) : 0;
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
