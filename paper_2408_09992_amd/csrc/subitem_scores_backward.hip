// Eq. 4's gradients (pq_subitem_scores_backward): for every split two small products with the tables' gradient,
//
//   dqueries[q][k s + e] = sum_j dS[q][k][j] psi[k][j][e]         dcentroids[k][j][e] = sum_q dS[q][k][j] phi[q][k s + e]
//
// on the fp32 matrix cores, both in one launch.
#include "pqtopk_train.h"
#include "head_common.hpp"

namespace pqk {
namespace head {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 512, kWaves = kThreads / kWave, kTile = 32;

struct GradArgs {
    const float *dS, *queries, *centroids;
    float *dqueries, *dcentroids;
    int B, d, m, b, s;
    int tiles_e, tiles_j, tiles_q;                   // tiles of 32 elements of a chunk, sub-ids, queries
    int centroid_blocks;                             // workgroups of dcentroids; those of dqueries come after them
    int vec;                                         // rows of dS are read as 16-byte vectors
};

// 32 x 32 partial products of the waves, added in the waves' order; element (row, col) goes to put(row, col, sum).
template <typename Put>
__device__ __forceinline__ void join_waves(const f32x16& acc, float (*part)[kTile * kTile], Put put) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
    for (int i = 0; i < 16; ++i) part[wave][(8 * (i / 4) + 4 * (lane / 32) + i % 4) * kTile + lane % 32] = acc[i];
    __syncthreads();
#pragma unroll
    for (int e = threadIdx.x; e < kTile * kTile; e += kThreads) {
        float sum = part[0][e];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) sum += part[w][e];
        put(e / kTile, e % kTile, sum);
    }
}

// A workgroup makes one 32 x 32 tile; its eight waves share the summed index and are joined through LDS.  Operands go from
// memory to the matrix cores' registers directly: a tile's rows are read once, in whole lines (rows of dS, of psi, of phi).
// Launch and latency bound up to some thousand queries (4 B b d flops are 0.5 GFLOP at 1024 queries, d = 512, b = 256).
__global__ __launch_bounds__(kThreads) void subitem_scores_backward_kernel(GradArgs a) {
    __shared__ float part[kWaves][kTile * kTile];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, col = lane % 32, half = lane / 32;
    f32x16 acc = {};
    const size_t table = (size_t)a.m * a.b;                    // floats of a query's tables
    if ((int)blockIdx.x < a.centroid_blocks) {
        int t = blockIdx.x;
        const int e0 = t % a.tiles_e * kTile; t /= a.tiles_e;
        const int j0 = t % a.tiles_j * kTile, k = t / a.tiles_j;
        const bool has_j = j0 + col < a.b, has_e = e0 + col < a.s;
        const float* dS = a.dS + (size_t)k * a.b + min(j0 + col, a.b - 1);
        const float* phi = a.queries + (size_t)k * a.s + min(e0 + col, a.s - 1);
        // a wave's step: queries 2 * (wave + kWaves * i) + half, sixteen loads ahead of their products
        constexpr int kSteps = 8;
        for (int q0 = 2 * wave; q0 < a.B; q0 += 2 * kWaves * kSteps) {
            float x[kSteps], y[kSteps];
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int q = q0 + 2 * kWaves * i + half, at = min(q, a.B - 1);
                x[i] = dS[(size_t)at * table];
                y[i] = phi[(size_t)at * a.d];
                x[i] = q < a.B && has_j ? x[i] : 0.0f;
                y[i] = q < a.B && has_e ? y[i] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < kSteps; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], acc, 0, 0, 0);
        }
        join_waves(acc, part, [&](int row, int c, float v) {
            if (j0 + row < a.b && e0 + c < a.s) a.dcentroids[((size_t)k * a.b + j0 + row) * a.s + e0 + c] = v;
        });
        return;
    }
    int t = blockIdx.x - a.centroid_blocks;
    const int e0 = t % a.tiles_e * kTile; t /= a.tiles_e;
    const int k = t % a.m, q0 = t / a.m * kTile;
    const bool has_q = q0 + col < a.B, has_e = e0 + col < a.s;
    const float* dS = a.dS + (size_t)min(q0 + col, a.B - 1) * table + (size_t)k * a.b;
    const float* psi = a.centroids + (size_t)k * a.b * a.s + min(e0 + col, a.s - 1);
    // a wave's step: sub-ids 8 (wave + kWaves i) .. + 7, of which a lane reads four in a row; any order of the summed index
    // will do as long as both operands follow it
    for (int j0 = 8 * wave; j0 < a.b; j0 += 8 * kWaves) {
        const int j = j0 + 4 * half;
        float x[4], y[4];
        if (a.vec && j + 4 <= a.b) {
            const float4 v = *reinterpret_cast<const float4*>(dS + j);
            x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = dS[min(j + i, a.b - 1)];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = psi[(size_t)min(j + i, a.b - 1) * a.s];
            x[i] = has_q && j + i < a.b ? x[i] : 0.0f;
            y[i] = has_e && j + i < a.b ? y[i] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], acc, 0, 0, 0);
    }
    join_waves(acc, part, [&](int row, int c, float v) {
        if (q0 + row < a.B && e0 + c < a.s) a.dqueries[(size_t)(q0 + row) * a.d + (size_t)k * a.s + e0 + c] = v;
    });
}

}  // namespace
}  // namespace head
}  // namespace pqk

using namespace pqk::head;

extern "C" int pq_subitem_scores_backward(const float* dS, const float* queries, const float* centroids, float* dqueries,
                                          float* dcentroids, int B, int d, int m, int b, void* stream) {
    if (!dS || (!dqueries && !dcentroids) || (dqueries && !centroids) || (dcentroids && !queries)) return PQ_ERR_NULL;
    if (B < 1 || d < 1 || m < 1 || b < 1 || b > 65536 || d % m != 0) return PQ_ERR_SHAPE;
    if (B > PQ_MAX_B || m > PQ_MAX_M) return PQ_ERR_UNSUPPORTED;
    if (((uintptr_t)dS | (uintptr_t)queries | (uintptr_t)centroids | (uintptr_t)dqueries | (uintptr_t)dcentroids) & 3) return PQ_ERR_ALIGN;
    GradArgs a{dS, queries, centroids, dqueries, dcentroids, B, d, m, b, d / m, 0, 0, 0, 0, 0};
    a.tiles_e = (int)ceil_div(a.s, kTile);
    a.tiles_j = (int)ceil_div(b, kTile);
    a.tiles_q = (int)ceil_div(B, kTile);
    a.vec = b % 4 == 0 && ((uintptr_t)dS & 15) == 0;
    const long long by_centroid = dcentroids ? (long long)a.tiles_e * a.tiles_j * m : 0, by_query = dqueries ? (long long)a.tiles_e * a.tiles_q * m : 0;
    if (by_centroid + by_query > 2147483647LL) return PQ_ERR_UNSUPPORTED;
    a.centroid_blocks = (int)by_centroid;
    hipLaunchKernelGGL(subitem_scores_backward_kernel, dim3((unsigned)(by_centroid + by_query)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
    return pqk::record_hip_error(hipGetLastError());
}
