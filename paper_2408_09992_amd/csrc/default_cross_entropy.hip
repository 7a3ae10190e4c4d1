// Softmax cross entropy of the catalogue by the default scorer's W phi (pq_default_cross_entropy), and its gradients.
//
//   z = H W^T      lse_t = log sum_i exp z_ti      dz_ti = g_t (exp(z_ti - lse_t) - [i = target_t])
//   dH = dz W      dW = dz^T H
//
// Everything is a matrix product whose one side is short: T positions, d elements, N items.  The loss keeps z in registers:
// a workgroup multiplies a tile of items by a tile of positions and folds it into the positions' running sums.  The gradient
// takes the items in pieces: z of a piece once more, its dz to a buffer that stays in the last-level cache, then the two
// products from there.  8 T N d operations in all, 2 of them the loss's.
#include <type_traits>
#include "pqtopk_train.h"
#include "matrix_tile.hpp"

namespace pqk {
namespace head {
namespace {

constexpr int kThreads = 256;
constexpr float kHeadroom = 40.0f;                    // (log2) how far a score may rise over a lane's reference before that moves
constexpr float kDzBits = 15.0f, kDzScale = 32768.0f;  // dz is stored times 2^15 over the largest |g|: types keep small probabilities
constexpr int kItems = 256;                           // items of a tile

struct RowInfo { float at, scale; };                  // of a position: 2^(z log2e - at) is p 2^15; its g over the largest |g|

// Which tiles: `wide` for more than 64 positions.
template <bool WIDE> struct Shape;
template <> struct Shape<true> {
    static constexpr int kPositions = 128;
    template <typename T> using Scores = MatrixTile<T, kItems, kPositions, 128, 64, true, true>;
    static constexpr int kRowsH = 256, kColsH = 128;  // dH
    template <typename T> using ProductH = MatrixTile<T, kRowsH, kColsH, 128, 64, true, false>;
};
template <> struct Shape<false> {
    static constexpr int kPositions = 64;
    template <typename T> using Scores = MatrixTile<T, kItems, kPositions, 64, 64, true, true>;
    static constexpr int kRowsH = 64, kColsH = 256;
    template <typename T> using ProductH = MatrixTile<T, kRowsH, kColsH, 64, 64, true, false>;
};
constexpr int kColsW = 128;                           // dW: items x elements
template <typename T> using ProductW = MatrixTile<T, kItems, kColsW, 128, 64, false, false>;

// Neighbouring workgroups run on different chiplets, each with its own L2: workgroup `id` of n per outer tile becomes
// (outer, inner) such that all inner tiles of an outer one follow each other on one chiplet and share its rows there.
__device__ __forceinline__ void chiplet_order(int id, int inner_tiles, int& outer, int& inner) {
    const int chiplet = id % 8, local = id / 8;
    inner = local % inner_tiles;
    outer = local / inner_tiles * 8 + chiplet;
}

// How many of a wave's `rows` rows there are, given how many follow its first one.
__device__ __forceinline__ int left_of(long long rest, int rows) { return (int)max(0LL, min(rest, (long long)rows)); }

struct DenseArgs {
    const void *W, *H;
    const int* targets;
    long long N;
    int B, d;
    // loss
    long long item_tiles;
    int tiles_each, groups, position_tiles;
    float2* partial;                                   // [groups][B]
    float *loss, *lse;
    // gradient
    const float *lse_in, *grad;
    RowInfo* info;                                     // [positions, padded]
    float* factor;                                     // what the products are multiplied with
    void* dz;                                          // [tiles of a piece][positions, padded][kItems]
    float* partial_h;                                  // [slices][B][d]
    void *dH, *dW;
    long long first_item;                              // of the piece
    int piece, items;                                  // padded and actual items of it
    int padded, slices, slice_items, more;             // positions padded; shares of a piece's items; partial_h holds earlier pieces
    int tiles_m, tiles_n;                              // of the launch
};

template <typename T>
__device__ __forceinline__ Operand items_of(const DenseArgs& a, long long item) {
    return Operand{a.W, (size_t)a.d * sizeof(T), item, a.N, 0, a.d};
}
template <typename T>
__device__ __forceinline__ Operand positions_of(const DenseArgs& a, int position) {
    return Operand{a.H, (size_t)a.d * sizeof(T), position, a.B, 0, a.d};
}

// Statistics of a tile of positions over a group of item tiles, one after the other.  As in the loss by sub-ids a lane's
// reference c moves only when a score passes it by 2^kHeadroom; lanes, halves and waves join once, at the end.
template <typename T, bool WIDE>
__global__ __launch_bounds__(kThreads, 2) void default_cross_entropy_kernel(DenseArgs a) {
    using Tile = typename Shape<WIDE>::template Scores<T>;
    constexpr int BN = Shape<WIDE>::kPositions, MI = Tile::MI, NI = Tile::NI, kRowWaves = kThreads / kWave * (NI * 32) / BN;
    __shared__ float2 stat[kRowWaves][BN];
    int group, pt;
    chiplet_order(blockIdx.x, a.position_tiles, group, pt);
    if (group >= a.groups) return;
    const int lane = threadIdx.x % kWave;
    float c[NI], s[NI];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) { c[ni] = -__builtin_inff(); s[ni] = 0.0f; }
    for (int i = 0; i < a.tiles_each; ++i) {
        const long long tile = (long long)group * a.tiles_each + i;
        if (tile >= a.item_tiles) break;
        f32x16 acc[MI][NI];
        Tile::run(items_of<T>(a, tile * kItems), positions_of<T>(a, pt * BN), acc);
        const int left = left_of(a.N - tile * kItems - Tile::wave_row(), 32 * MI);
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) {
            __builtin_amdgcn_sched_barrier(0);                 // (one column after the other: the registers hold no two of them)
            float top = -__builtin_inff();
            if (left < 32 * MI) {
                stay_a_branch();
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (32 * mi + 8 * (e / 4) + e % 4 >= left - 4 * (lane / 32)) acc[mi][ni][e] = -__builtin_inff();
            }
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, acc[mi][ni][e]);
            top *= kLog2e;
            if (__any(top > c[ni] + kHeadroom)) {
                if (top > c[ni] + kHeadroom) { s[ni] *= exp2_fast(c[ni] - top); c[ni] = top; }
            }
            const float at = c[ni] == -__builtin_inff() ? 0.0f : c[ni];
            float sum = 0.0f;
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum += exp2_fast(fmaf(acc[mi][ni][e], kLog2e, -at));
            s[ni] += sum;
        }
    }
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
        const float c2 = __shfl_xor(c[ni], 32), s2 = __shfl_xor(s[ni], 32);
        join_sums(c[ni], s[ni], c2, s2);
        if (lane < 32) stat[Tile::wave_row() / (32 * MI)][Tile::wave_col() + 32 * ni + lane] = make_float2(c[ni], s[ni]);
    }
    __syncthreads();
    const int q = pt * BN + threadIdx.x;
    if ((int)threadIdx.x < BN && q < a.B) {
        float2 t = stat[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < kRowWaves; ++w) join_sums(t.x, t.y, stat[w][threadIdx.x].x, stat[w][threadIdx.x].y);
        a.partial[(size_t)group * a.B + q] = t;
    }
}

// One wave per position joins the groups' sums and takes the target's score.
template <typename T>
__global__ __launch_bounds__(kWave) void default_cross_entropy_join_kernel(DenseArgs a) {
    const int q = blockIdx.x, lane = threadIdx.x;
    float c = -__builtin_inff(), s = 0.0f;
    for (int i = lane; i < a.groups; i += kWave) {
        const float2 t = a.partial[(size_t)i * a.B + q];
        join_sums(c, s, t.x, t.y);
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) {
        const float c2 = __shfl_xor(c, x), s2 = __shfl_xor(s, x);
        join_sums(c, s, c2, s2);
    }
    const float lse = (c + __log2f(s)) * kLn2;
    const int t = a.targets[q];
    float z = 0.0f;
    const bool has = t >= 0 && t < a.N;
    if (has) {
        const T *w = static_cast<const T*>(a.W) + (size_t)t * a.d, *h = static_cast<const T*>(a.H) + (size_t)q * a.d;
        for (int e = lane; e < a.d; e += kWave) z = fmaf((float)w[e], (float)h[e], z);
#pragma unroll
        for (int x = 1; x < kWave; x *= 2) z += __shfl_xor(z, x);
    }
    if (lane == 0) {
        a.lse[q] = lse;
        a.loss[q] = has ? lse - z : 0.0f;
    }
}

// What the gradient's kernels need of a position, and the factor of their products.
__global__ __launch_bounds__(1024) void default_rows_kernel(DenseArgs a) {
    __shared__ float tops[16];
    const int tid = threadIdx.x;
    auto weight = [&](int q) { const int t = a.targets[q]; return t >= 0 && t < a.N ? a.grad[q] : 0.0f; };
    float top = 0.0f;
    for (int q = tid; q < a.B; q += 1024) top = fmaxf(top, fabsf(weight(q)));
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
    if (tid % kWave == 0) tops[tid / kWave] = top;
    __syncthreads();
    top = tops[0];
#pragma unroll
    for (int w = 1; w < 16; ++w) top = fmaxf(top, tops[w]);
    for (int q = tid; q < a.padded; q += 1024) {
        const float g = q < a.B ? weight(q) : 0.0f;
        const bool live = g != 0.0f;
        a.info[q] = RowInfo{live ? a.lse_in[q] * kLog2e - kDzBits : __builtin_inff(), live ? g / top : 0.0f};
    }
    if (tid == 0) *a.factor = top / kDzScale;
}

// dz of a piece of items: scores as in the loss, then (exp(z - lse) - [target]) g as the products' operands, position by
// position.  For 16-bit operands dz is rounded to their type: it is the products' input as H and W are, and what they add up
// (in float32) is rounded to that type once more at the end.
template <typename T, bool WIDE>
__global__ __launch_bounds__(kThreads, 2) void default_dz_kernel(DenseArgs a) {
    using Tile = typename Shape<WIDE>::template Scores<T>;
    constexpr int BN = Shape<WIDE>::kPositions, MI = Tile::MI, NI = Tile::NI;
    int tile, pt;
    chiplet_order(blockIdx.x, a.tiles_n, tile, pt);
    if (tile >= a.tiles_m) return;
    const int lane = threadIdx.x % kWave;
    const long long item0 = a.first_item + (long long)tile * kItems;
    f32x16 acc[MI][NI];
    Tile::run(items_of<T>(a, item0), positions_of<T>(a, pt * BN), acc);
    const int left = left_of(a.N - item0 - Tile::wave_row(), 32 * MI) - 4 * (lane / 32);
    unsigned char* own = Tile::own_memory();
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
        const int q0 = pt * BN + Tile::wave_col() + 32 * ni, q = q0 + lane % 32;
        const RowInfo info = a.info[q];
        const long long from_first = (q < a.B ? (long long)a.targets[q] : -1) - item0 - Tile::wave_row();
        const int hit = from_first >= 0 && from_first < 32 * MI ? (int)from_first - 4 * (lane / 32) : -64;
        const bool special = __any(hit > -64) || left < 32 * MI - 4;           // (rare: a target among these items, the catalogue's end)
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[mi][ni][e] = exp2_fast(fmaf(acc[mi][ni][e], kLog2e, -info.at));
        if (special) {
            stay_a_branch();
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int at = 32 * mi + 8 * (e / 4) + e % 4;
                    if (at == hit) acc[mi][ni][e] -= kDzScale;
                    if (at >= left) acc[mi][ni][e] = 0.0f;
                }
        }
        // 32 positions x 32 items at a time through the wave's LDS: positions leave in rows of 16-byte pieces.  The pieces of
        // a row are swapped by its number, so that writes and reads spread over the banks.
        constexpr int kPieces = 32 * (int)sizeof(T) / 16;
        T* out = static_cast<T*>(a.dz) + ((size_t)tile * a.padded + q0) * kItems + Tile::wave_row();
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            typedef T T4 __attribute__((ext_vector_type(4)));
#pragma unroll
            for (int four = 0; four < 4; ++four) {
                T4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (T)(acc[mi][ni][4 * four + e] * info.scale);
                const int byte = (8 * four + 4 * (lane / 32)) * (int)sizeof(T), piece = (byte / 16) ^ (lane % 32 / (8 / kPieces) % kPieces);
                *reinterpret_cast<T4*>(own + (lane % 32 * kPieces + piece) * 16 + byte % 16) = v;
            }
            wave_reads_after_writes();
#pragma unroll
            for (int i = 0; i < kPieces / 2; ++i) {
                const int at = i * kWave + lane, row = at / kPieces, piece = at % kPieces;
                const uint4 v = *reinterpret_cast<const uint4*>(own + (row * kPieces + (piece ^ (row / (8 / kPieces) % kPieces))) * 16);
                *reinterpret_cast<uint4*>(reinterpret_cast<unsigned char*>(out + (size_t)row * kItems + 32 * mi) + piece * 16) = v;
            }
            wave_reads_after_writes();
        }
    }
}

// dW of a piece: [items][d], summed over the positions.
template <typename T>
__global__ __launch_bounds__(kThreads, 2) void default_dw_kernel(DenseArgs a) {
    using Tile = ProductW<T>;
    int tile, ct;
    chiplet_order(blockIdx.x, a.tiles_n, tile, ct);
    if (tile >= a.tiles_m) return;
    const int lane = threadIdx.x % kWave;
    f32x16 acc[Tile::MI][Tile::NI];
    const Operand dz{static_cast<const T*>(a.dz) + (size_t)tile * a.padded * kItems, kItems * sizeof(T), 0, kItems, 0, a.padded};
    const Operand h{a.H, (size_t)a.d * sizeof(T), (long long)ct * kColsW, a.d, 0, a.B};
    Tile::run(dz, h, acc);
    const float factor = *a.factor;
    const long long item0 = a.first_item + (long long)tile * kItems + Tile::wave_row();
    const int left = left_of(a.N - item0, 32 * Tile::MI), col0 = ct * kColsW + Tile::wave_col();
    // 32 items x 32 elements at a time through the wave's LDS, as in default_dz_kernel
    constexpr int kPieces = 32 * (int)sizeof(T) / 16;
    unsigned char* own = Tile::own_memory();
#pragma unroll
    for (int mi = 0; mi < Tile::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < Tile::NI; ++ni) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int row = 8 * (e / 4) + 4 * (lane / 32) + e % 4, byte = lane % 32 * (int)sizeof(T);
                const int piece = (byte / 16) ^ (row / (8 / kPieces) % kPieces);
                *reinterpret_cast<T*>(own + (row * kPieces + piece) * 16 + byte % 16) = (T)(acc[mi][ni][e] * factor);
            }
            wave_reads_after_writes();
#pragma unroll
            for (int i = 0; i < kPieces / 2; ++i) {
                const int at = i * kWave + lane, row = at / kPieces, piece = at % kPieces;
                const uint4 v = *reinterpret_cast<const uint4*>(own + (row * kPieces + (piece ^ (row / (8 / kPieces) % kPieces))) * 16);
                const int col = col0 + 32 * ni + piece * (16 / (int)sizeof(T));
                if (32 * mi + row < left && col < a.d)
                    *reinterpret_cast<uint4*>(static_cast<T*>(a.dW) + (size_t)(item0 + 32 * mi + row) * a.d + col) = v;
            }
            wave_reads_after_writes();
        }
}

// A slice's share of dH: [positions][d] summed over its items of the piece, added to what earlier pieces left there.
template <typename T, bool WIDE>
__global__ __launch_bounds__(kThreads, 2) void default_dh_kernel(DenseArgs a) {
    using Tile = typename Shape<WIDE>::template ProductH<T>;
    constexpr int BM = Shape<WIDE>::kRowsH, BN = Shape<WIDE>::kColsH;
    int slice, tile;
    chiplet_order(blockIdx.x, a.tiles_m * a.tiles_n, slice, tile);
    if (slice >= a.slices) return;
    const int rt = tile / a.tiles_n, ct = tile % a.tiles_n;
    const int lane = threadIdx.x % kWave;
    const long long k0 = min((long long)slice * a.slice_items, (long long)a.items), k1 = min(k0 + a.slice_items, (long long)a.items);
    if (a.more && k0 == k1) return;
    f32x16 acc[Tile::MI][Tile::NI];
    const Operand dz{a.dz, kItems * sizeof(T), (long long)rt * BM, a.padded, k0, k1, kItems, (size_t)a.padded * kItems * sizeof(T)};
    const Operand w{static_cast<const T*>(a.W) + (size_t)a.first_item * a.d, (size_t)a.d * sizeof(T), (long long)ct * BN, a.d, k0,
                    min(k1, a.N - a.first_item)};
    if (k0 < k1) Tile::run(dz, w, acc);
    else {
#pragma unroll
        for (int mi = 0; mi < Tile::MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < Tile::NI; ++ni) acc[mi][ni] = f32x16{};
    }
    const int q0 = rt * BM + Tile::wave_row(), left = left_of(a.B - q0, 32 * Tile::MI) - 4 * (lane / 32);
    float* out = a.partial_h + ((size_t)slice * a.B + q0 + 4 * (lane / 32)) * a.d;
    auto put = [&](auto whole_c) {
        constexpr bool whole = decltype(whole_c)::value;
#pragma unroll
        for (int mi = 0; mi < Tile::MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < Tile::NI; ++ni) {
                const int col = ct * BN + Tile::wave_col() + 32 * ni + lane % 32;
                float* p = out + (size_t)(32 * mi) * a.d + min(col, a.d - 1);
                auto row = [&](int e) { return 32 * mi + 8 * (e / 4) + e % 4; };
                float old[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) old[e] = 0.0f;
                if (a.more && (whole || left > 32 * mi)) {         // (all of them asked for at once; past the end the first row's)
#pragma unroll
                    for (int e = 0; e < 16; ++e) old[e] = p[(size_t)(whole || row(e) < left ? row(e) - 32 * mi : 0) * a.d];
                }
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (col < a.d && (whole || row(e) < left)) p[(size_t)(row(e) - 32 * mi) * a.d] = old[e] + acc[mi][ni][e];
            }
    };
    if (a.B - q0 >= 32 * Tile::MI) put(std::true_type{});
    else put(std::false_type{});
}

// The slices' shares of dH, added in their order.
template <typename T>
__global__ __launch_bounds__(256) void default_dh_join_kernel(DenseArgs a) {
    const size_t n = (size_t)a.B * a.d, i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float sum = a.partial_h[i];
    for (int s = 1; s < a.slices; ++s) sum += a.partial_h[(size_t)s * n + i];
    static_cast<T*>(a.dH)[i] = (T)(sum * *a.factor);
}

// ---------------------------------------------------------------------------------------------------------------
// host side

struct DensePlan {
    bool wide;
    int position_tiles, tiles_each, groups;            // loss
    long long item_tiles;
    int piece, pieces, padded, slices, rows_tiles, cols_tiles;   // gradient
    size_t info_at, dz_at, partial_at, bytes;          // its workspace
};

constexpr long long kDzElements = 1LL << 27;           // of the buffer: 256 MB of 16-bit dz, the size of the last-level cache
constexpr long long kMaxPiece = 1LL << 22;

DensePlan plan_dense(long long N, int B, int d, int size) {
    DensePlan p;
    p.wide = B > 64;
    const int bn = p.wide ? 128 : 64;
    p.position_tiles = (int)ceil_div(B, bn);
    p.item_tiles = ceil_div(N, kItems);
    // two workgroups a compute unit and four rounds of them, if there are that many tiles
    const long long wanted = ceil_div(2LL * kCUs * 4, p.position_tiles);
    p.tiles_each = (int)ceil_div(p.item_tiles, wanted < 1 ? 1 : wanted);
    p.groups = (int)ceil_div(p.item_tiles, p.tiles_each);
    p.padded = p.position_tiles * bn;
    long long piece = kDzElements / p.padded;
    if (piece < 2048) piece = 2048;
    if (piece > kMaxPiece) piece = kMaxPiece;
    p.pieces = (int)ceil_div(N, piece);
    p.piece = (int)round_up((size_t)ceil_div(N, p.pieces), kItems);
    p.pieces = (int)ceil_div(N, p.piece);
    p.rows_tiles = (int)ceil_div(p.padded, p.wide ? 256 : 64);
    p.cols_tiles = (int)ceil_div(d, p.wide ? 128 : 256);
    long long slices = 2LL * kCUs / ((long long)p.rows_tiles * p.cols_tiles);
    const long long most = p.piece / kItems;
    p.slices = (int)(slices < 1 ? 1 : slices > most ? most : slices);
    p.info_at = 256;
    p.dz_at = round_up(p.info_at + (size_t)p.padded * sizeof(RowInfo), 256);
    p.partial_at = round_up(p.dz_at + (size_t)p.padded * p.piece * size, 256);
    p.bytes = round_up(p.partial_at + (size_t)p.slices * B * d * sizeof(float), 256);
    return p;
}

int size_of(int type) { return type == PQ_FLOAT32 ? 4 : type == PQ_BFLOAT16 || type == PQ_FLOAT16 ? 2 : 0; }

int check_dense(long long N, int B, int d, int type) {
    if (N < 1 || B < 1 || d < 1 || N >= 2147483648LL || size_of(type) == 0) return PQ_ERR_SHAPE;
    if (B > PQ_MAX_B || d > 16384 || d % (16 / size_of(type)) != 0) return PQ_ERR_UNSUPPORTED;
    return PQ_OK;
}

int grid_of(long long outer, long long inner) { return (int)(ceil_div(outer, 8) * 8 * inner); }     // see chiplet_order()

template <typename T, bool WIDE>
hipError_t run_loss(const DensePlan& p, const DenseArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((default_cross_entropy_kernel<T, WIDE>), dim3(grid_of(p.groups, p.position_tiles)), dim3(kThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((default_cross_entropy_join_kernel<T>), dim3(a.B), dim3(kWave), 0, st, a);
    return hipGetLastError();
}

template <typename T, bool WIDE>
hipError_t run_backward(const DensePlan& p, DenseArgs a, hipStream_t st) {
    hipLaunchKernelGGL(default_rows_kernel, dim3(1), dim3(1024), 0, st, a);
    hipError_t e = hipGetLastError();
    for (int i = 0; i < p.pieces && e == hipSuccess; ++i) {
        a.first_item = (long long)i * p.piece;
        const long long left = a.N - a.first_item;
        a.items = (int)round_up((size_t)(left < p.piece ? left : p.piece), kItems);
        a.more = i > 0;
        const int tiles = a.items / kItems;
        DenseArgs s = a;
        s.tiles_m = tiles;
        s.tiles_n = p.position_tiles;
        hipLaunchKernelGGL((default_dz_kernel<T, WIDE>), dim3(grid_of(tiles, p.position_tiles)), dim3(kThreads), 0, st, s);
        if ((e = hipGetLastError()) != hipSuccess) break;
        s.tiles_n = (int)ceil_div(a.d, kColsW);
        hipLaunchKernelGGL((default_dw_kernel<T>), dim3(grid_of(tiles, s.tiles_n)), dim3(kThreads), 0, st, s);
        if ((e = hipGetLastError()) != hipSuccess) break;
        s.tiles_m = p.rows_tiles;
        s.tiles_n = p.cols_tiles;
        s.slice_items = (int)round_up((size_t)ceil_div(a.items, p.slices), kItems);
        hipLaunchKernelGGL((default_dh_kernel<T, WIDE>), dim3(grid_of(p.slices, p.rows_tiles * p.cols_tiles)), dim3(kThreads), 0, st, s);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((default_dh_join_kernel<T>), dim3((unsigned)ceil_div((long long)a.B * a.d, 256)), dim3(256), 0, st, a);
    return hipGetLastError();
}

size_t loss_bytes(const DensePlan& p, int B) { return round_up((size_t)p.groups * B * sizeof(float2), 16); }

}  // namespace
}  // namespace head
}  // namespace pqk

using namespace pqk::head;

extern "C" {

size_t pq_default_cross_entropy_workspace_bytes(long long N, int B, int d, int type) {
    return check_dense(N, B, d, type) == PQ_OK ? loss_bytes(plan_dense(N, B, d, size_of(type)), B) : 0;
}

int pq_default_cross_entropy(const void* W, const void* queries, const int* targets, long long N, int B, int d, int type, float* loss,
                             float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!W || !queries || !targets || !loss || !lse || !workspace) return PQ_ERR_NULL;
    const int rc = check_dense(N, B, d, type);
    if (rc != PQ_OK) return rc;
    if ((((uintptr_t)W | (uintptr_t)queries | (uintptr_t)workspace) & 15) || (((uintptr_t)targets | (uintptr_t)loss | (uintptr_t)lse) & 3)) return PQ_ERR_ALIGN;
    const DensePlan p = plan_dense(N, B, d, size_of(type));
    if (workspace_bytes < loss_bytes(p, B)) return PQ_ERR_WORKSPACE;
    DenseArgs a{};
    a.W = W; a.H = queries; a.targets = targets; a.N = N; a.B = B; a.d = d;
    a.item_tiles = p.item_tiles; a.tiles_each = p.tiles_each; a.groups = p.groups; a.position_tiles = p.position_tiles;
    a.partial = static_cast<float2*>(workspace); a.loss = loss; a.lse = lse;
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (type == PQ_FLOAT32) e = p.wide ? run_loss<float, true>(p, a, st) : run_loss<float, false>(p, a, st);
    else if (type == PQ_BFLOAT16) e = p.wide ? run_loss<__bf16, true>(p, a, st) : run_loss<__bf16, false>(p, a, st);
    else e = p.wide ? run_loss<_Float16, true>(p, a, st) : run_loss<_Float16, false>(p, a, st);
    return pqk::record_hip_error(e);
}

size_t pq_default_cross_entropy_backward_workspace_bytes(long long N, int B, int d, int type) {
    return check_dense(N, B, d, type) == PQ_OK ? plan_dense(N, B, d, size_of(type)).bytes : 0;
}

int pq_default_cross_entropy_backward(const void* W, const void* queries, const int* targets, const float* lse, const float* grad_loss,
                                      long long N, int B, int d, int type, void* dqueries, void* dW, void* workspace,
                                      size_t workspace_bytes, void* stream) {
    if (!W || !queries || !targets || !lse || !grad_loss || !dqueries || !dW || !workspace) return PQ_ERR_NULL;
    const int rc = check_dense(N, B, d, type);
    if (rc != PQ_OK) return rc;
    if ((((uintptr_t)W | (uintptr_t)queries | (uintptr_t)workspace) & 15) ||
        (((uintptr_t)targets | (uintptr_t)lse | (uintptr_t)grad_loss) & 3) || (((uintptr_t)dqueries | (uintptr_t)dW) & 15))
        return PQ_ERR_ALIGN;
    const DensePlan p = plan_dense(N, B, d, size_of(type));
    if (workspace_bytes < p.bytes) return PQ_ERR_WORKSPACE;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    DenseArgs a{};
    a.W = W; a.H = queries; a.targets = targets; a.N = N; a.B = B; a.d = d;
    a.lse_in = lse; a.grad = grad_loss; a.dH = dqueries; a.dW = dW;
    a.factor = reinterpret_cast<float*>(ws);
    a.info = reinterpret_cast<RowInfo*>(ws + p.info_at);
    a.dz = ws + p.dz_at;
    a.partial_h = reinterpret_cast<float*>(ws + p.partial_at);
    a.piece = p.piece; a.padded = p.padded; a.slices = p.slices;
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (type == PQ_FLOAT32) e = p.wide ? run_backward<float, true>(p, a, st) : run_backward<float, false>(p, a, st);
    else if (type == PQ_BFLOAT16) e = p.wide ? run_backward<__bf16, true>(p, a, st) : run_backward<__bf16, false>(p, a, st);
    else e = p.wide ? run_backward<_Float16, true>(p, a, st) : run_backward<_Float16, false>(p, a, st);
    return pqk::record_hip_error(e);
}

}  // extern "C"
