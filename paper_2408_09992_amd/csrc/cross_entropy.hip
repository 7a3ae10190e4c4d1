// pq_cross_entropy* and their gradients: launches and entry points (the kernels and plans: cross_entropy.hpp).
#include "cross_entropy.hpp"

namespace pqk {
namespace head {
namespace subids {
namespace {

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

template <int M, typename CT, int Q>
hipError_t go_loss(const Plan& p, const LossArgs& a, hipStream_t st) {
    hipError_t e = allow_lds(cross_entropy_kernel<M, CT, Q>, p.lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((cross_entropy_kernel<M, CT, Q>), dim3(p.shares, p.groups), dim3(kThreads), p.lds, st, a);
    return hipGetLastError();
}
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
hipError_t go_loss_m(const Plan& p, const LossArgs& a, hipStream_t st) {
    if (a.m == 4) return go_loss_q<4, CT>(p, a, st);
    if (a.m == 8) return go_loss_q<8, CT>(p, a, st);
    if (a.m == 16) return go_loss_q<16, CT>(p, a, st);
    if (a.m == 2 && sizeof(CT) == 1) return go_loss_q<2, uint8_t>(p, a, st);
    if (a.m == 32 && sizeof(CT) == 1) return go_loss_q<32, uint8_t>(p, a, st);
    if (a.m == 64 && sizeof(CT) == 1) return go_loss_q<64, uint8_t>(p, a, st);
    return go_loss_q<0, CT>(p, a, st);
}
template <typename CT>
hipError_t go_backward_m(const Plan& p, const BackArgs& a, hipStream_t st) {
    if (a.m == 4) return go_backward_q<4, CT>(p, a, st);
    if (a.m == 8) return go_backward_q<8, CT>(p, a, st);
    if (a.m == 16) return go_backward_q<16, CT>(p, a, st);
    if (a.m == 2 && sizeof(CT) == 1) return go_backward_q<2, uint8_t>(p, a, st);
    if (a.m == 32 && sizeof(CT) == 1) return go_backward_q<32, uint8_t>(p, a, st);
    if (a.m == 64 && sizeof(CT) == 1) return go_backward_q<64, uint8_t>(p, a, st);
    return go_backward_q<0, CT>(p, a, st);
}

}  // namespace

hipError_t launch_loss(const Plan& p, const LossArgs& a, int code_bytes, hipStream_t st) {
    return code_bytes == 1 ? go_loss_m<uint8_t>(p, a, st) : go_loss_m<uint16_t>(p, a, st);
}
hipError_t launch_backward(const Plan& p, const BackArgs& a, int code_bytes, int shares, hipStream_t st) {
    const hipError_t e = code_bytes == 1 ? go_backward_m<uint8_t>(p, a, st) : go_backward_m<uint16_t>(p, a, st);
    if (e != hipSuccess || shares == 1) return e;
    const size_t entries = (size_t)a.B * a.m * a.b;
    if (shares > kJoinLeads)
        hipLaunchKernelGGL(cross_entropy_backward_join_kernel<kJoinLeads>, dim3((unsigned)ceil_div(entries, kJoinThreads / kJoinLeads)), dim3(kJoinThreads), 0, st, a, shares, code_bytes);
    else
        hipLaunchKernelGGL(cross_entropy_backward_join_kernel<1>, dim3((unsigned)ceil_div(entries, kJoinThreads)), dim3(kJoinThreads), 0, st, a, shares, code_bytes);
    return hipGetLastError();
}

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
    hipError_t e = launch_loss(p, a, sizeof(CT), st);
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
    BackArgs a{codes, S, targets, lse, grad, N, B, m, b, p.kept, p.share, static_cast<uint64_t*>(ws), dS, nullptr, kLog2e};
    return record_hip_error(launch_backward(p, a, sizeof(CT), p.shares, st));
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
