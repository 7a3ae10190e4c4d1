// pq_cross_entropy* and their gradients: launches and entry points (the kernels and plans: cross_entropy.hpp).
#include "cross_entropy.hpp"

namespace pqk {
namespace head {
namespace subids {
namespace {

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
    LossArgs a{codes, S, targets, N, B, m, b, p.share, static_cast<float2*>(ws), out, lse, kLog2e};
    return record_hip_error(launch_loss<CT>(p, a, st));
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
    BackArgs a{codes, S, targets, lse, grad, N, B, m, b, p.kept, p.share, static_cast<uint64_t*>(ws), dS, kLog2e, (double)kLog2e};
    return record_hip_error(launch_backward<CT>(p, a, st));
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
}  // namespace subids
}  // namespace head
}  // namespace pqk

using namespace pqk::head::subids;

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
