// Eq. 4's gradients (pq_subitem_scores_backward): for every split two small products with the tables' gradient,
//
//   dqueries[q][k s + e] = sum_j dS[q][k][j] psi[k][j][e]         dcentroids[k][j][e] = sum_q dS[q][k][j] phi[q][k s + e]
//
// on the fp32 matrix cores, both in one launch.
#include "pqtopk_train.h"
#include "matrix_tile.hpp"

namespace pqk {
namespace head {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / kWave, kTile = 32;

struct GradArgs {
    const float *dS, *queries, *centroids;
    float *dqueries, *dcentroids;
    int B, d, m, b, s;
    int tiles_e, tiles_j, tiles_q;                   // tiles of 32 elements of a chunk, sub-ids, queries
    int centroid_blocks;                             // workgroups of dcentroids; those of dqueries come after them
    int vec;                                         // rows of dS are read as 16-byte vectors
    // by tiles of 64 x 64
    int shares, share;                               // of the queries that a tile of dcentroids is summed over
    float* partial;                                  // [shares][m][b][s], if there are more than one
};

// 32 x 32 partial products of the waves, added in the waves' order; element (row, col) goes to put(row, col, sum).
template <typename Put>
__device__ __forceinline__ void join_waves(const f32x16& acc, float (*part)[kTile * kTile], Put put) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
    for (int i = 0; i < 16; ++i) part[wave][(8 * (i / 4) + 4 * (lane / 32) + i % 4) * kTile + lane % 32] = acc[i];
    __syncthreads();
    for (int e = threadIdx.x; e < kTile * kTile; e += kThreads) {
        float sum = part[0][e];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) sum += part[w][e];
        put(e / kTile, e % kTile, sum);
    }
}

// Few queries, or rows that are not whole 16-byte pieces.  A workgroup makes one 32 x 32 tile; its eight waves share the summed
// index and are joined through LDS.  Operands go from memory to the matrix cores' registers directly: a tile's rows are read
// once, in whole lines (rows of dS, of psi, of phi).  Bound by the latency of these loads: 4.8 us for one query, 6.5 for 256 and
// 27 for 2048 (d = 512, m = 8, b = 256), where the tiles below take 17.6.
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
        // a wave's step: queries 2 * (wave + kWaves * i) + half, eight of them; the loads of the next two steps are under way
        constexpr int kSteps = 8, kStride = 2 * kWaves * kSteps, kAhead = 2;
        float nx[kAhead][kSteps], ny[kAhead][kSteps];
        auto load = [&](int slot, int q0) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int at = min(q0 + 2 * kWaves * i + half, a.B - 1);
                nx[slot][i] = dS[(size_t)at * table];
                ny[slot][i] = phi[(size_t)at * a.d];
            }
        };
#pragma unroll
        for (int slot = 0; slot < kAhead; ++slot) load(slot, 2 * wave + slot * kStride);
        for (int base = 0; base < a.B; base += kAhead * kStride) {
#pragma unroll
            for (int slot = 0; slot < kAhead; ++slot) {
                const int q0 = base + 2 * wave + slot * kStride;
                float x[kSteps], y[kSteps];
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const bool there = q0 + 2 * kWaves * i + half < a.B;
                    x[i] = there && has_j ? nx[slot][i] : 0.0f;
                    y[i] = there && has_e ? ny[slot][i] : 0.0f;
                }
                if (base + kAhead * kStride < a.B) load(slot, q0 + kAhead * kStride);
#pragma unroll
                for (int i = 0; i < kSteps; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], acc, 0, 0, 0);
            }
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
    constexpr int kAhead = 4;                                  // steps whose loads are under way
    float x[kAhead][4], y[kAhead][4];
    auto load = [&](int slot, int j) {
        if (a.vec && j + 4 <= a.b) {
            const float4 v = *reinterpret_cast<const float4*>(dS + j);
            x[slot][0] = v.x; x[slot][1] = v.y; x[slot][2] = v.z; x[slot][3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[slot][i] = dS[min(j + i, a.b - 1)];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) y[slot][i] = psi[(size_t)min(j + i, a.b - 1) * a.s];
    };
    const int j_first = 8 * wave + 4 * half, j_stride = 8 * kWaves;
#pragma unroll
    for (int s = 0; s < kAhead; ++s) load(s, j_first + s * j_stride);
    for (int j0 = 0; j0 < a.b; j0 += kAhead * j_stride) {      // (the same rounds for all lanes: past the last sub-id zeros)
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
            const int j = j_first + j0 + s * j_stride;
            float u[4], v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u[i] = has_q && j + i < a.b ? x[s][i] : 0.0f;
                v[i] = has_e && j + i < a.b ? y[s][i] : 0.0f;
            }
            if (j0 + kAhead * j_stride < a.b) load(s, j + kAhead * j_stride);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(u[i], v[i], acc, 0, 0, 0);
        }
    }
    join_waves(acc, part, [&](int row, int c, float v) {
        if (q0 + row < a.B && e0 + c < a.s) a.dqueries[(size_t)(q0 + row) * a.d + (size_t)k * a.s + e0 + c] = v;
    });
}

// Many queries: tiles of 64 x 64 through LDS (matrix_tile.hpp), those of dcentroids summed over a share of the queries each.
// Products of float32 in three bfloat16 pieces a factor.  8192 queries (d = 512, m = 8, b = 256; 84 MB of tables and queries):
// 43 us, 2.0 TB/s (40 without the join); fewer are bound by the latency of a share's few stages and of the second launch.
using TileQ = MatrixTile<float, 64, 64, 32, 32, true, false>;
using TileC = MatrixTile<float, 64, 64, 32, 32, false, false>;
constexpr int kSide = 64;

__global__ __launch_bounds__(TileQ::kThreads) void subitem_scores_backward_tiles_kernel(GradArgs a) {
    const int lane = threadIdx.x % kWave;
    const size_t table_bytes = (size_t)a.m * a.b * sizeof(float), row_bytes = (size_t)a.d * sizeof(float);
    f32x16 acc[1][1];
    if ((int)blockIdx.x < a.centroid_blocks) {
        int t = blockIdx.x;
        const int e0 = t % a.tiles_e * kSide; t /= a.tiles_e;
        const int j0 = t % a.tiles_j * kSide; t /= a.tiles_j;
        const int k = t % a.m, share = t / a.m;
        const long long q0 = (long long)share * a.share, q1 = min(q0 + a.share, (long long)a.B);
        TileC::run(Operand{a.dS + (size_t)k * a.b, table_bytes, j0, a.b, q0, q1}, Operand{a.queries + (size_t)k * a.s, row_bytes, e0, a.s, q0, q1}, acc);
        float* out = (a.shares > 1 ? a.partial + (size_t)share * a.m * a.b * a.s : a.dcentroids) + (size_t)k * a.b * a.s;
        const int e = e0 + TileC::wave_col() + lane % 32;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int j = j0 + TileC::wave_row() + 8 * (i / 4) + 4 * (lane / 32) + i % 4;
            if (j < a.b && e < a.s) out[(size_t)j * a.s + e] = acc[0][0][i];
        }
        return;
    }
    int t = blockIdx.x - a.centroid_blocks;
    const int e0 = t % a.tiles_e * kSide; t /= a.tiles_e;
    const int k = t % a.m;
    const int q0 = t / a.m * kSide;
    TileQ::run(Operand{a.dS + (size_t)k * a.b, table_bytes, q0, a.B, 0, a.b}, Operand{a.centroids + (size_t)k * a.b * a.s, (size_t)a.s * sizeof(float), e0, a.s, 0, a.b}, acc);
    const int e = e0 + TileQ::wave_col() + lane % 32;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int q = q0 + TileQ::wave_row() + 8 * (i / 4) + 4 * (lane / 32) + i % 4;
        if (q < a.B && e < a.s) a.dqueries[(size_t)q * a.d + (size_t)k * a.s + e] = acc[0][0][i];
    }
}

// The shares of dcentroids, added in their order.
__global__ __launch_bounds__(256) void subitem_scores_backward_join_kernel(GradArgs a) {
    const size_t n = (size_t)a.m * a.b * a.s, i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float sum = a.partial[i];
#pragma unroll 8
    for (int s = 1; s < a.shares; ++s) sum += a.partial[(size_t)s * n + i];
    a.dcentroids[i] = sum;
}

// From how many queries on the tiles pay (both ways, d = 512, m = 8, b = 256: 256 queries 6.6 us without them, 10.0 with;
// 1024 15.4 and 15.6; 2048 27.2 and 17.5; 8192 97 and 43).
constexpr int kTilesMinQueries = 1024;
// Shares of the queries: as many as bring workgroups for half the chip, of 128 queries at least.
int shares_of(int B, int m, int b, int s) {
    const long long tiles = (long long)m * ceil_div(b, kSide) * ceil_div(s, kSide);
    long long shares = ceil_div(kCUs, tiles);
    if (shares > B / 128) shares = B / 128;
    return (int)(shares < 1 ? 1 : shares);
}

int check_backward(int B, int d, int m, int b) {
    if (B < 1 || d < 1 || m < 1 || b < 1 || b > 65536 || d % m != 0) return PQ_ERR_SHAPE;
    return B > PQ_MAX_B || m > PQ_MAX_M ? PQ_ERR_UNSUPPORTED : PQ_OK;
}

size_t backward_bytes(int B, int d, int m, int b) {
    const int shares = B >= kTilesMinQueries ? shares_of(B, m, b, d / m) : 1;
    return round_up((shares > 1 ? (size_t)shares * b * d * sizeof(float) : 0) + 16, 16);
}

}  // namespace
}  // namespace head
}  // namespace pqk

using namespace pqk::head;

extern "C" size_t pq_subitem_scores_backward_workspace_bytes(int B, int d, int m, int b) {
    return check_backward(B, d, m, b) == PQ_OK ? backward_bytes(B, d, m, b) : 0;
}

extern "C" int pq_subitem_scores_backward(const float* dS, const float* queries, const float* centroids, float* dqueries,
                                          float* dcentroids, int B, int d, int m, int b, void* workspace, size_t workspace_bytes,
                                          void* stream) {
    if (!dS || !workspace || (!dqueries && !dcentroids) || (dqueries && !centroids) || (dcentroids && !queries)) return PQ_ERR_NULL;
    const int rc = check_backward(B, d, m, b);
    if (rc != PQ_OK) return rc;
    if ((((uintptr_t)dS | (uintptr_t)queries | (uintptr_t)centroids | (uintptr_t)dqueries | (uintptr_t)dcentroids) & 3) || ((uintptr_t)workspace & 15))
        return PQ_ERR_ALIGN;
    if (workspace_bytes < backward_bytes(B, d, m, b)) return PQ_ERR_WORKSPACE;
    GradArgs a{};
    a.dS = dS; a.queries = queries; a.centroids = centroids; a.dqueries = dqueries; a.dcentroids = dcentroids;
    a.B = B; a.d = d; a.m = m; a.b = b; a.s = d / m;
    // (the tiles' loads are of 16 bytes)
    const bool tiles = B >= kTilesMinQueries && b % 4 == 0 && a.s % 4 == 0 && (((uintptr_t)dS | (uintptr_t)queries | (uintptr_t)centroids) & 15) == 0;
    const int side = tiles ? kSide : kTile;
    a.tiles_e = (int)ceil_div(a.s, side);
    a.tiles_j = (int)ceil_div(b, side);
    a.tiles_q = (int)ceil_div(B, side);
    a.vec = b % 4 == 0 && ((uintptr_t)dS & 15) == 0;
    a.shares = tiles && dcentroids ? shares_of(B, m, b, a.s) : 1;
    a.share = (int)ceil_div(B, a.shares);
    a.shares = (int)ceil_div(B, a.share);
    a.partial = static_cast<float*>(workspace);
    const long long by_centroid = dcentroids ? (long long)a.tiles_e * a.tiles_j * m * a.shares : 0, by_query = dqueries ? (long long)a.tiles_e * a.tiles_q * m : 0;
    if ((by_centroid + by_query) * (tiles ? (int)TileQ::kThreads : kThreads) > 0xFFFFFFFFLL) return PQ_ERR_UNSUPPORTED;       // (a launch's threads)
    a.centroid_blocks = (int)by_centroid;
    const dim3 grid((unsigned)(by_centroid + by_query));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (tiles) hipLaunchKernelGGL(subitem_scores_backward_tiles_kernel, grid, dim3(TileQ::kThreads), 0, st, a);
    else hipLaunchKernelGGL(subitem_scores_backward_kernel, grid, dim3(kThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.shares > 1) {
        hipLaunchKernelGGL(subitem_scores_backward_join_kernel, dim3((unsigned)ceil_div((long long)b * d, 256)), dim3(256), 0, st, a);
        e = hipGetLastError();
    }
    return pqk::record_hip_error(e);
}
