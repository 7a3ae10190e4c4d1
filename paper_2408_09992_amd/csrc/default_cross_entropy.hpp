// Softmax cross entropy of the catalogue by the default scorer's W phi (pq_default_cross_entropy), and its gradients.
//
//   z = H W^T      lse_t = log sum_i exp z_ti      dz_ti = g_t (exp(z_ti - lse_t) - [i = target_t])
//   dH = dz W      dW = dz^T H
//
// Everything is a matrix product whose one side is short: T positions, d elements, N items.  The loss keeps z in registers:
// a workgroup multiplies a tile of items by a tile of positions and folds it into the positions' running sums.  The gradient
// takes the items in pieces: z of a piece once more, its dz to a buffer, then the two products from there.  8 T N d operations
// in all, 2 of them the loss's.
#pragma once
#include <type_traits>
#include "pqtopk_train.h"
#include "matrix_tile.hpp"

namespace pqk {
namespace head {

constexpr float kHeadroom = 40.0f;                    // (log2) how far a score may rise over a lane's reference before that moves
constexpr float kDzBits = 15.0f, kDzScale = 32768.0f;  // dz is stored times 2^15 over a weight (RowInfo): types keep small probabilities
constexpr int kItems = 256;                           // items of a block of dz, and of most tiles of z and dW

// Of a row of dz: 2^(z log2e - at) is p 2^15; its g over what dz is stored over; what its row of dH is multiplied with.  dz is stored over
// the largest |g| of all positions, but in float16, whose exponents would not reach far below that (a position of a millionth of the
// largest weight would keep probabilities down to 2^-19 alone), over that times a power of two of the position's own: what is left
// of its weight is over a half, and 1 where all weights are the same.  (Over powers of two alone the same mantissa would be rounded in all
// rows, and with it the whole gradient be off by up to a unit.)
struct RowInfo { float at, scale, factor; };
template <typename T> constexpr bool kOwnPowers = std::is_same<T, _Float16>::value;

// The tiles: z for ITEMS items and POS positions; dH for ROWS positions and COLS elements; dW for ITEMS items and COLS
// elements.  Tiles of 256 x 256 by eight waves feed the matrix cores best (208 TFLOP/s in float32, 1040 to 1130 in bfloat16,
// against 203 and 880 to 1090 with 256 x 128 by four); the smaller ones are for few positions and narrow embeddings.  Those of
// 64 x 64 are for products that do not fill the chip: it is the latency of a tile's stages that bounds them, and the share of the
// memory's rate that few compute units have.
template <typename T, int POS, int ITEMS> struct ScoresTile;
template <typename T> struct ScoresTile<T, 64, 64> : MatrixTile<T, 64, 64, 32, 32, true, true> {};
template <typename T> struct ScoresTile<T, 64, 256> : MatrixTile<T, 256, 64, 64, 64, true, true> {};
template <typename T> struct ScoresTile<T, 128, 256> : MatrixTile<T, 256, 128, 128, 64, true, true> {};
template <typename T> struct ScoresTile<T, 256, 256> : MatrixTile<T, 256, 256, 128, 64, true, true> {};
template <typename T, int COLS, int ITEMS> struct TileW;
template <typename T> struct TileW<T, 64, 64> : MatrixTile<T, 64, 64, 32, 32, false, false> {};
template <typename T> struct TileW<T, 64, 256> : MatrixTile<T, 64, 256, 64, 64, false, false> {};
template <typename T> struct TileW<T, 128, 256> : MatrixTile<T, 128, 256, 128, 64, false, false> {};
template <typename T> struct TileW<T, 256, 256> : MatrixTile<T, 256, 256, 128, 64, false, false> {};
template <typename T, int ROWS, int COLS> struct TileH;
template <typename T> struct TileH<T, 64, 64> : MatrixTile<T, 64, 64, 32, 32, true, false> {};
template <typename T> struct TileH<T, 64, 128> : MatrixTile<T, 64, 128, 32, 64, true, false> {};
template <typename T> struct TileH<T, 64, 256> : MatrixTile<T, 64, 256, 64, 64, true, false> {};
template <typename T> struct TileH<T, 128, 64> : MatrixTile<T, 128, 64, 64, 32, true, false> {};
template <typename T> struct TileH<T, 128, 128> : MatrixTile<T, 128, 128, 64, 64, true, false> {};
template <typename T> struct TileH<T, 128, 256> : MatrixTile<T, 128, 256, 64, 128, true, false> {};
template <typename T> struct TileH<T, 256, 64> : MatrixTile<T, 256, 64, 64, 64, true, false> {};
template <typename T> struct TileH<T, 256, 128> : MatrixTile<T, 256, 128, 128, 64, true, false> {};
template <typename T> struct TileH<T, 256, 256> : MatrixTile<T, 256, 256, 128, 64, true, false> {};

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
    int parts;                                         // rows of dz that a position has (see dz_rows)
    RowInfo* info;                                     // [rows of dz, padded]
    void* live;                                        // [rows of dz][d]: the queries, zeros where a position adds nothing
    float* factor;                                     // what dW is multiplied with
    int* block_powers;                                 // float16: of the blocks of default_rows_kernel, see scale_rows_kernel
    void* scaled;                                      // float16: [rows of dz][d], the queries that dW is made of
    void* dz;                                          // [tiles of a piece][rows of dz, padded][kItems]
    float* partial_h;                                  // [slices][rows of dz][d]
    void *dH, *dW;
    long long first_item;                              // of the piece
    int piece, items;                                  // padded and actual items of it
    int padded, slices, slice_items, more;             // rows of dz padded; shares of a piece's items; partial_h holds earlier pieces
    int tiles_m, tiles_n;                              // of the launch
    int h_rows, h_cols, w_blocks;                      // tiles of dH; workgroups that make dW, where one launch makes both
};

template <typename T>
__device__ __forceinline__ Operand items_of(const DenseArgs& a, long long item) {
    return Operand{a.W, (size_t)a.d * sizeof(T), item, a.N, 0, a.d};
}
template <typename T>
__device__ __forceinline__ Operand positions_of(const DenseArgs& a, int position) {
    return Operand{a.H, (size_t)a.d * sizeof(T), position, a.B, 0, a.d};
}

// dz in 16 bits has two rows a position where there are up to 32 positions, B rounded values and then B of what their rounding
// leaves.  A row of dqueries is then (and a row of dW may be) little more than one value of dz times one row, whose error that
// rounding would double (one position, 17,902 items of 64 float16: dW 4.4e-5 off instead of 2.8e-5).  Tiles have 64 rows anyway.  With more
// positions the errors of their rows are independent: together with the result's own rounding at most sqrt(2) of it in the mean square.
// (Positions that share a weight share its rounding too, where it is no power of two of the largest.)
constexpr int kTwoParts = 32;
__device__ __forceinline__ int dz_rows(const DenseArgs& a) { return a.B * a.parts; }
__device__ __forceinline__ int position_of(const DenseArgs& a, int row) { return row < a.B ? row : row - a.B; }

// Statistics of a tile of positions over a group of item tiles, one after the other.  As in the loss by sub-ids a lane's
// reference c moves only when a score passes it by 2^kHeadroom; lanes, halves and waves join once, at the end.
// Bound by the matrix cores: 1024 positions, 1.28M items of 512 bfloat16, 1.44 to 1.56 ms, 860 to 930 TFLOP/s with an exponential
// per score; 2048 positions, 34,742 items of 512 float32, 404 to 439 us, 166 to 181 TFLOP/s (4.25 rounds of tiles).
template <typename T, int BN, int ITEMS>
__global__ __launch_bounds__((ScoresTile<T, BN, ITEMS>::kThreads), 2) void default_cross_entropy_kernel(DenseArgs a) {
    using Tile = ScoresTile<T, BN, ITEMS>;
    constexpr int MI = Tile::MI, NI = Tile::NI, kRowWaves = ITEMS / (32 * MI);
    __shared__ float2 stat[kRowWaves][BN];
    int group, pt;
    chiplet_order(blockIdx.x, a.position_tiles, group, pt);
    if (group >= a.groups) return;
    const int lane = threadIdx.x % kWave;
    float c[NI], s[NI];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) { c[ni] = kLowest; s[ni] = 0.0f; }
    for (int i = 0; i < a.tiles_each; ++i) {
        const long long tile = (long long)group * a.tiles_each + i;
        if (tile >= a.item_tiles) break;
        f32x16 acc[MI][NI];
        Tile::run(items_of<T>(a, tile * ITEMS), positions_of<T>(a, pt * BN), acc);
        const int left = left_of(a.N - tile * ITEMS - Tile::wave_row(), 32 * MI);
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
                if (top > c[ni] + kHeadroom) raise_reference(c[ni], s[ni], top);
            }
            float sum = 0.0f;
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum += exp2_fast(fmaf(acc[mi][ni][e], kLog2e, -c[ni]));
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
    float c = kLowest, s = 0.0f;
    for (int i = lane; i < a.groups; i += kWave) {
        const float2 t = a.partial[(size_t)i * a.B + q];
        join_sums(c, s, t.x, t.y);
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) {
        const float c2 = __shfl_xor(c, x), s2 = __shfl_xor(s, x);
        join_sums(c, s, c2, s2);
    }
    const float lse = log_sum(c, s);
    const int t = a.targets[q];
    float z = 0.0f;
    const bool has = t >= 0 && t < a.N && lse != -__builtin_inff();
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

__device__ __forceinline__ float wave_top(float v) {
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) v = fmaxf(v, __shfl_xor(v, x));
    return v;
}
// The power of two above |x|, x a number but 0: |x| 2^-power is at least a half.
__device__ __forceinline__ int power_of(float x) {
    int e;
    (void)frexpf(x, &e);
    return e;
}
// The power of two that a weight over the largest is more than half of, and at most; 0 where it is no number.
__device__ __forceinline__ int weight_power(float over_top) {
    if (!(fabsf(over_top) < __builtin_inff())) return 0;
    int e;
    return frexpf(fabsf(over_top), &e) == 0.5f ? e - 1 : e;
}
// What a number is to the largest of its kind: an infinite one is none.  (As a weight it would be what all other positions are stored over.)
__device__ __forceinline__ float weight_size(float g) { return fabsf(g) < __builtin_inff() ? fabsf(g) : 0.0f; }
// Of a position with gradient g (0: it adds nothing), the largest of all being top.
template <typename T>
__device__ __forceinline__ RowInfo row_info(float g, float top, float lse) {
    if (g == 0.0f) return RowInfo{__builtin_inff(), 0.0f, 0.0f};
    if constexpr (kOwnPowers<T>) {
        const int power = weight_power(g / top);
        return RowInfo{lse * kLog2e - kDzBits, ldexpf(g / top, -power), top * ldexpf(1.0f / kDzScale, power)};
    } else return RowInfo{lse * kLog2e - kDzBits, g / top, top / kDzScale};
}

// The share of the gradient of a row's position: 0 where there is none, no target, no item in play or no position.
__device__ __forceinline__ float row_weight(const DenseArgs& a, int row) {
    const int q = min(position_of(a, row), a.B - 1), t = a.targets[q];
    const float g = a.grad[q], lse = a.lse_in[q];              // (all three asked for at once)
    return row < dz_rows(a) && t >= 0 && t < a.N && lse != -__builtin_inff() ? g : 0.0f;
}
// The queries in pieces of 16 bytes, from piece `first` on every `stride`-th, with zeros for positions that add nothing.
// Float16: returns the power of two above these pieces' largest product of a query's element and its position's power.
constexpr int kNoPower = -100000;
template <typename T>
__device__ __forceinline__ int copy_live(const DenseArgs& a, size_t first, size_t stride, float top = 0.0f) {
    const int row_pieces = a.d * (int)sizeof(T) / 16;
    const size_t pieces = (size_t)dz_rows(a) * row_pieces, position_pieces = (size_t)a.B * row_pieces;
    int power = kNoPower;
    for (size_t i = first; i < pieces; i += stride) {
        uint4 v = static_cast<const uint4*>(a.H)[i < position_pieces ? i : i - position_pieces];
        const float g = row_weight(a, (int)(i / row_pieces));
        if (g == 0.0f) v = uint4{0, 0, 0, 0};
        static_cast<uint4*>(a.live)[i] = v;
        if constexpr (kOwnPowers<T>) {
            const f16x8 h = __builtin_bit_cast(f16x8, v);
            float largest = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) largest = fmaxf(largest, weight_size((float)h[e]));
            if (largest > 0.0f) power = max(power, weight_power(g / top) + power_of(largest));
        }
    }
    return power;
}
__device__ __forceinline__ int wave_max(int v) {
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) v = max(v, __shfl_xor(v, x));
    return v;
}

// What the gradient's kernels need of a position, the factor of their products, and the queries they multiply: those of a
// position without a target (padding: it may hold anything, NaN too) are zeros, as 0 NaN would be NaN in every dW.
// A copy of the queries is B d elements beside the N d that the products read.
template <typename T>
__global__ __launch_bounds__(1024) void default_rows_kernel(DenseArgs a) {
    __shared__ float tops[16];
    __shared__ int powers[16];
    const int tid = threadIdx.x;
    const size_t first = (size_t)blockIdx.x * 1024 + tid, stride = (size_t)gridDim.x * 1024;
    if constexpr (!kOwnPowers<T>) {
        copy_live<T>(a, first, stride);
        if (blockIdx.x != 0) return;
    }
    float top = 0.0f;
    for (int q = tid; q < a.B; q += 1024) top = fmaxf(top, weight_size(row_weight(a, q)));
    top = wave_top(top);
    if (tid % kWave == 0) tops[tid / kWave] = top;
    __syncthreads();
    top = tops[0];
#pragma unroll
    for (int w = 1; w < 16; ++w) top = fmaxf(top, tops[w]);
    if constexpr (kOwnPowers<T>) {
        int power = wave_max(copy_live<T>(a, first, stride, top));
        if (tid % kWave == 0) powers[tid / kWave] = power;
        __syncthreads();
        if (tid < kWave) {
            power = wave_max(powers[tid % 16]);
            if (tid == 0) a.block_powers[blockIdx.x] = power;
        }
        if (blockIdx.x != 0) return;
    }
    for (int q = tid; q < a.padded; q += 1024) {
        a.info[q] = row_info<T>(row_weight(a, q), top, a.lse_in[min(position_of(a, q), a.B - 1)]);
    }
    if (tid == 0) a.factor[kOwnPowers<T> ? 1 : 0] = kOwnPowers<T> ? top : top / kDzScale;
}

// Float16: the queries that dW is made of, each times the power of two that its position's dz was stored over, and all times the one that
// brings the largest below 2^15 (factor[1]: the largest weight).  So what float16 cannot hold of a small weight's queries is 2^-40 of the largest product of weight and query.
template <typename T>
__global__ __launch_bounds__(1024) void scale_rows_kernel(DenseArgs a) {
    const int lane = threadIdx.x % kWave;
    int power = kNoPower;
    for (int i = lane; i < (int)gridDim.x; i += kWave) power = max(power, a.block_powers[i]);          // (as many blocks made them)
    power = wave_max(power);
    const float top = a.factor[1];
    const int row_pieces = a.d * (int)sizeof(T) / 16;
    const size_t pieces = (size_t)dz_rows(a) * row_pieces;
    for (size_t i = (size_t)blockIdx.x * 1024 + threadIdx.x; i < pieces; i += (size_t)gridDim.x * 1024) {
        f16x8 h = static_cast<const f16x8*>(a.live)[i];
        const float g = row_weight(a, (int)(i / row_pieces));
        const int by = g == 0.0f ? 0 : weight_power(g / top) + 15 - power;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = (_Float16)ldexpf((float)h[e], by);
        static_cast<f16x8*>(a.scaled)[i] = h;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.factor = power == kNoPower ? 0.0f : ldexpf(top, power - 30);
}

// Blocks of 32 x 32 results leave through the wave's LDS, N of them at a time, in rows of 16-byte pieces: row lane % 32 of a block
// is a column of the product, element 8 (e / 4) + 4 (lane / 32) + e % 4 of it is value(block, e), and put(block, row, piece, its
// 16 bytes) takes them on.  The pieces of a row are swapped by its number, so that writes and reads spread over the banks.
template <typename T, int MI> constexpr int kBlocks = sizeof(T) == 2 && MI % 2 == 0 ? 2 : 1;          // (4 KB a wave)
template <int N, typename Value, typename Put>
__device__ __forceinline__ void store_blocks(unsigned char* own, Value value, Put put) {
    typedef decltype(value(0, 0)) T;
    typedef T T4 __attribute__((ext_vector_type(4)));
    constexpr int kPieces = 32 * (int)sizeof(T) / 16, kBytes = 32 * 32 * (int)sizeof(T);
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int four = 0; four < 4; ++four) {
            T4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = value(k, 4 * four + e);
            const int byte = (8 * four + 4 * (lane / 32)) * (int)sizeof(T), piece = (byte / 16) ^ (lane % 32 / (8 / kPieces) % kPieces);
            *reinterpret_cast<T4*>(own + k * kBytes + (lane % 32 * kPieces + piece) * 16 + byte % 16) = v;
        }
    wave_reads_after_writes();
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < kPieces / 2; ++i) {
            const int at = i * kWave + lane, row = at / kPieces, piece = at % kPieces;
            put(k, row, piece, *reinterpret_cast<const uint4*>(own + k * kBytes + (row * kPieces + (piece ^ (row / (8 / kPieces) % kPieces))) * 16));
        }
    wave_reads_after_writes();
}

// dz of a piece of items: scores as in the loss, then (exp(z - lse) - [target]) g as the products' operands, position by
// position.  For 16-bit operands dz is rounded to their type: it is the products' input as H and W are, and what they add up
// (in float32) is rounded to that type once more at the end (up to 32 positions keep what the first rounding leaves: kTwoParts).
// 131,072 items, 1024 positions of 512 bfloat16: 179 to 187 us, 750 TFLOP/s, and 268 MB written.
// ROWS: up to 64 rows of dz, whose info (see default_rows_kernel) the workgroups make themselves.
template <typename T, int BN, int ITEMS, bool ROWS>
__global__ __launch_bounds__((ScoresTile<T, BN, ITEMS>::kThreads), 2) void default_dz_kernel(DenseArgs a) {
    using Tile = ScoresTile<T, BN, ITEMS>;
    constexpr int MI = Tile::MI, NI = Tile::NI;
    static_assert(!ROWS || BN == kWave, "a row is a lane");
    static_assert(!ROWS || !kOwnPowers<T>, "scale_rows_kernel comes after default_rows_kernel");
    constexpr bool kParts = BN == kWave && sizeof(T) == 2;     // (whether there may be two a position)
    int tile, pt;
    chiplet_order(blockIdx.x, a.tiles_n, tile, pt);
    if (tile >= a.tiles_m) return;
    const int lane = threadIdx.x % kWave;
    RowInfo own_row{};
    if constexpr (ROWS) {                                      // (every wave: lane r has row r's)
        const float g = row_weight(a, lane);
        const float top = wave_top(weight_size(g));
        own_row = row_info<T>(g, top, a.lse_in[min(position_of(a, lane), a.B - 1)]);
        if (!a.more) {
            copy_live<T>(a, (size_t)tile * Tile::kThreads + threadIdx.x, (size_t)a.tiles_m * Tile::kThreads);
            if (tile == 0 && threadIdx.x < kWave) a.info[lane] = own_row;
            if (tile == 0 && threadIdx.x == 0) *a.factor = top / kDzScale;
        }
    }
    const long long item0 = a.first_item + (long long)tile * ITEMS;
    f32x16 acc[MI][NI];
    Operand positions = positions_of<T>(a, pt * BN);
    if constexpr (kParts) positions.again = a.parts > 1 ? a.B : 0;
    Tile::run(items_of<T>(a, item0), positions, acc);
    const int left = left_of(a.N - item0 - Tile::wave_row(), 32 * MI) - 4 * (lane / 32);
    unsigned char* own = Tile::own_memory();
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
        const int q0 = pt * BN + Tile::wave_col() + 32 * ni, q = q0 + lane % 32;
        RowInfo info;
        if constexpr (ROWS) info = RowInfo{__shfl(own_row.at, q0 + lane % 32), __shfl(own_row.scale, q0 + lane % 32)};
        else info = a.info[q];
        const bool rest = kParts && q >= a.B;
        const long long from_first = (q < (kParts ? dz_rows(a) : a.B) ? (long long)a.targets[rest ? q - a.B : q] : -1) - item0 - Tile::wave_row();
        const int hit = from_first >= 0 && from_first < 32 * MI ? (int)from_first - 4 * (lane / 32) : -64;
        const bool special = __any(hit > -64) || left < 32 * MI - 4;           // (rare: a target among these items, the catalogue's end)
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float p = exp2_fast(fmaf(acc[mi][ni][e], kLog2e, -info.at));
                acc[mi][ni][e] = ROWS && info.at == __builtin_inff() ? 0.0f : p;       // (its query may be NaN: not a copy that is zeros)
            }
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
        if constexpr (kParts) {
            if (a.parts > 1) {
                stay_a_branch();
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float x = acc[mi][ni][e] * info.scale;
                        acc[mi][ni][e] = rest ? fmaf(acc[mi][ni][e], info.scale, -(float)(T)x) : x;
                    }
                info.scale = 1.0f;
            }
        }
        T* out = static_cast<T*>(a.dz) + ((size_t)(tile / (kItems / ITEMS)) * a.padded + q0) * kItems + tile % (kItems / ITEMS) * ITEMS + Tile::wave_row();
#pragma unroll
        for (int mi = 0; mi < MI; mi += kBlocks<T, MI>)
            store_blocks<kBlocks<T, MI>>(own, [&](int k, int e) { return (T)(acc[mi + k][ni][e] * info.scale); },
                                         [&](int k, int row, int piece, uint4 v) {
                                             *reinterpret_cast<uint4*>(reinterpret_cast<unsigned char*>(out + (size_t)row * kItems + 32 * (mi + k)) + piece * 16) = v;
                                         });
    }
}

// A tile of dW of a piece: [items][d], summed over dz's rows.  As many: 133 to 145 us, about 1000 TFLOP/s.
template <typename T, int COLS, int ITEMS>
__device__ __forceinline__ void dw_tile(const DenseArgs& a, int block) {
    using Tile = TileW<T, COLS, ITEMS>;
    int tile, ct;
    chiplet_order(block, a.tiles_n, tile, ct);
    if (tile >= a.tiles_m) return;
    f32x16 acc[Tile::MI][Tile::NI];
    const Operand dz{static_cast<const T*>(a.dz) + (size_t)(tile / (kItems / ITEMS)) * a.padded * kItems, kItems * sizeof(T), tile % (kItems / ITEMS) * ITEMS, kItems, 0, a.padded};
    const Operand h{a.H, (size_t)a.d * sizeof(T), (long long)ct * COLS, a.d, 0, dz_rows(a)};
    Tile::run(h, dz, acc);                             // (elements by items: a lane has four neighbouring elements of an item)
    const float factor = *a.factor;
    const long long item0 = a.first_item + (long long)tile * ITEMS + Tile::wave_col();
    const int left = left_of(a.N - item0, 32 * Tile::NI), col0 = ct * COLS + Tile::wave_row();
    unsigned char* own = Tile::own_memory();
    constexpr int kOf = kBlocks<T, Tile::MI>;
#pragma unroll
    for (int ni = 0; ni < Tile::NI; ++ni)
#pragma unroll
        for (int mi = 0; mi < Tile::MI; mi += kOf)
            store_blocks<kOf>(own, [&](int k, int e) { return (T)(acc[mi + k][ni][e] * factor); },
                              [&](int k, int row, int piece, uint4 v) {
                                  const int col = col0 + 32 * (mi + k) + piece * (16 / (int)sizeof(T));
                                  if (32 * ni + row < left && col < a.d)
                                      *reinterpret_cast<uint4*>(static_cast<T*>(a.dW) + (size_t)(item0 + 32 * ni + row) * a.d + col) = v;
                              });
}

template <typename T, int COLS, int ITEMS>
__global__ __launch_bounds__((TileW<T, COLS, ITEMS>::kThreads), 2) void default_dw_kernel(DenseArgs a) { dw_tile<T, COLS, ITEMS>(a, blockIdx.x); }

// A slice's share of a tile of dH: [rows of dz][d] summed over its items of the piece, added to what earlier pieces left there.
// As many: 139 to 145 us, about 960 TFLOP/s.
template <typename T, int BM, int BN>
__device__ __forceinline__ void dh_tile(const DenseArgs& a, int block) {
    using Tile = TileH<T, BM, BN>;
    int slice, tile;
    chiplet_order(block, a.h_rows * a.h_cols, slice, tile);
    if (slice >= a.slices) return;
    const int rt = tile / a.h_cols, ct = tile % a.h_cols;
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
    const int rows = dz_rows(a), q0 = rt * BM + Tile::wave_row(), left = left_of(rows - q0, 32 * Tile::MI) - 4 * (lane / 32);
    float* out = a.partial_h + ((size_t)slice * rows + q0 + 4 * (lane / 32)) * a.d;
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
    if (rows - q0 >= 32 * Tile::MI) put(std::true_type{});
    else put(std::false_type{});
}
template <typename T, int BM, int BN>
__global__ __launch_bounds__((TileH<T, BM, BN>::kThreads), 2) void default_dh_kernel(DenseArgs a) { dh_tile<T, BM, BN>(a, blockIdx.x); }

// Both, by tiles of 64 x 64, where neither fills the chip and a launch takes as long as they do (10,000 items of 64, 50 positions
// in float32: 6.4 us, and the step 29 us instead of 34).
template <typename T>
__global__ __launch_bounds__((TileW<T, 64, 64>::kThreads), 2) void default_products_kernel(DenseArgs a) {
    if ((int)blockIdx.x < a.w_blocks) dw_tile<T, 64, 64>(a, blockIdx.x);
    else dh_tile<T, 64, 64>(a, blockIdx.x - a.w_blocks);
}

// ---------------------------------------------------------------------------------------------------------------
// Gradients for up to 64 positions of 16-bit operands, d <= 512: one pass over W.  With so few positions all three products of
// a tile of items are done before the memory has brought the next one, so a workgroup takes the tile from LDS for z, for dH
// and (as H lies there too) dW, and W is read once instead of twice, dz never leaves the chip.

constexpr int kFew = 64, kFewThreads = 512, kFewBytes = 32768;         // positions; threads; bytes of a tile of W

// Rows of CHUNKS 16-byte chunks in LDS, chunk c of row r at c ^ turn(r): sixteen rows' reads of one chunk (an operand with k
// along the rows) meet different banks, and so do four rows' reads of four (k across them, transposed).
template <int CHUNKS>
struct Rows {
    static constexpr int kBytes = CHUNKS * 16;
    static __device__ __forceinline__ int turn(int row) {
        return CHUNKS >= 16 ? row % 4 * 4 + row / 4 % 4 : CHUNKS == 8 ? row / 2 % 2 * 4 + row / 4 % 4 : row / 4 % 4;
    }
    static __device__ __forceinline__ int at(int row, int chunk) { return row * kBytes + ((chunk ^ turn(row)) * 16); }
    static __device__ __forceinline__ s16x8 along(const unsigned char* p, int row, int chunk) { return *reinterpret_cast<const s16x8*>(p + at(row, chunk)); }
    // of k0 .. k0 + 15 (stored rows) and 32 columns from col0 the lane's operand: column lane % 32, k 8 (lane / 32) .. + 7
    static __device__ __forceinline__ s16x8 across(const unsigned char* p, int k0, int col0) {
        const int lane = threadIdx.x % kWave, k = k0 + 8 * (lane / 32) + lane % 16 / 4, col = col0 + 16 * (lane / 16 % 2) + 4 * (lane % 4);
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + at(k, col / 8) + col % 8 * 2));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + at(k + 4, col / 8) + col % 8 * 2));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

typedef float f32x4_t __attribute__((ext_vector_type(4)));
template <typename T>
__device__ __forceinline__ f32x4_t multiply16(s16x8 x, s16x8 y, f32x4_t c) {
    if constexpr (std::is_same<T, __bf16>::value) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
}

// Rows of W or of the queries from `row0` on into LDS: LOADS 16-byte pieces a thread; past the last row the last one again
// (from the again-th, if not 0, the first ones), past a row's end zeros.
template <typename T, int D, int LOADS>
__device__ __forceinline__ void bring_rows(const void* base, int d, long long row0, long long rows, unsigned char* to, int again = 0) {
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const size_t ld = (size_t)d * sizeof(T);
    const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base)) + (size_t)row0 * ld, 0, kBufferBytes, 0x00020000);
    const int last = (int)min(rows - row0, 65536LL) - 1;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int piece = (wave * LOADS + i) * kWave + lane, row = piece / (D / 8), chunk = (piece % (D / 8)) ^ Rows<D / 8>::turn(row);
        const uint32_t offset = chunk * 8 < d ? (uint32_t)min(again && row >= again ? row - again : row, last) * (uint32_t)ld + (uint32_t)chunk * 16u : kPastEnd;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to + (wave * LOADS + i) * kWave * 16), 16, offset, 0, 0, 0);
    }
}

// The loss of up to 64 positions of 16-bit operands, d <= 512: as default_few_kernel below takes its tiles, so that loads do not
// pause between them (64 positions, 1.3 GB of W: 250 to 262 us, 5.0 to 5.2 TB/s; 271 by default_cross_entropy_kernel's tiles).
template <typename T, int D>
__global__ __launch_bounds__(kFewThreads, 2) void default_few_loss_kernel(DenseArgs a) {
    constexpr int IT = kFewBytes / 2 / D, kWaves = kFewThreads / kWave;
    using RowsD = Rows<D / 8>;
    __shared__ __align__(16) unsigned char w0[kFewBytes], w1[kFewBytes], h[kFew * D * 2];
    __shared__ float2 stat[kWaves][kFew];
    constexpr int kLoadsW = kFewBytes / 16 / kFewThreads, kLoadsH = kFew * D * 2 / 16 / kFewThreads;
    constexpr int kBlocksZ = IT / 16 * 4 / kWaves, kParts = kBlocksZ < 4 ? kBlocksZ : 4;       // a wave's blocks of 16 x 16; positions among them / 16
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const long long tiles = (a.N + IT - 1) / IT;
    bring_rows<T, D, kLoadsH>(a.H, a.d, 0, a.B, h);
    bring_rows<T, D, kLoadsW>(a.W, a.d, (long long)blockIdx.x * IT, a.N, w0);
    float c[kParts], s[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) { c[i] = kLowest; s[i] = 0.0f; }
    int turn = 0;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x, ++turn) {
        const unsigned char* w = turn % 2 ? w1 : w0;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");       // the tile has come, its other buffer is free
        bring_rows<T, D, kLoadsW>(a.W, a.d, min(tile + gridDim.x, tiles - 1) * IT, a.N, turn % 2 ? w0 : w1);
#pragma unroll
        for (int i = 0; i < kBlocksZ; ++i) {
            const int block = wave * kBlocksZ + i, item0 = block / 4 * 16, pos = block % 4 * 16 + lane % 16;
            f32x4_t z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
                z = multiply16<T>(RowsD::along(w, item0 + lane % 16, 4 * k + lane / 16), RowsD::along(h, pos, 4 * k + lane / 16), z);
            const int left = left_of(a.N - tile * IT - item0, 16) - lane / 16 * 4;
            if (left < 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e >= left) z[e] = -__builtin_inff();
            }
            const float top = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])) * kLog2e;
            const int part = i % kParts;
            if (__any(top > c[part] + kHeadroom)) {
                if (top > c[part] + kHeadroom) raise_reference(c[part], s[part], top);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[part] += exp2_fast(fmaf(z[e], kLog2e, -c[part]));
        }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");                  // (a last load into LDS may be under way)
    for (int q = lane; q < kFew; q += kWave) stat[wave][q] = make_float2(kLowest, 0.0f);
    wave_reads_after_writes();
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
#pragma unroll
        for (int x = 16; x < kWave; x *= 2) {
            const float c2 = __shfl_xor(c[i], x), s2 = __shfl_xor(s[i], x);
            join_sums(c[i], s[i], c2, s2);
        }
        if (lane < 16) stat[wave][(wave * kBlocksZ + i) % 4 * 16 + lane] = make_float2(c[i], s[i]);
    }
    __syncthreads();
    if (tid < a.B) {
        float2 t = stat[0][tid];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) join_sums(t.x, t.y, stat[w][tid].x, stat[w][tid].y);
        a.partial[(size_t)blockIdx.x * a.B + tid] = t;
    }
}

// D: d rounded up to 64, 128, 256 or 512.  A tile holds 16384 / D items.  Bound by memory: W in, dW out, 2.6 GB for 1.27M items
// of 512 elements in 515 to 550 us, 4.7 to 5.1 TB/s, where a copy reaches 4.73.
// PARTS: two rows of dz a position (kTwoParts), in the place of the other 32 positions.
template <typename T, int D, bool PARTS>
__global__ __launch_bounds__(kFewThreads, 2) void default_few_kernel(DenseArgs a) {
    constexpr int IT = kFewBytes / 2 / D, kWaves = kFewThreads / kWave;
    using RowsD = Rows<D / 8>;                                 // W and H
    using RowsI = Rows<IT / 8>;                                // dz: [row][item]
    __shared__ __align__(16) unsigned char w0[kFewBytes], w1[kFewBytes], h[kFew * D * 2], dz[kFew * IT * 2];
    // float16: dH's rows are stored over their own weights, for dW all over the largest
    constexpr bool kOwn = kOwnPowers<T>;
    __shared__ __align__(16) unsigned char dz_over_top[kOwn ? kFew * IT * 2 : 16];
    __shared__ float over_top[kFew];
    unsigned char* dz_w = kOwn ? dz_over_top : dz;
    __shared__ RowInfo info[kFew];
    __shared__ int target[kFew];
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const long long tiles = (a.N + IT - 1) / IT;
    constexpr int kLoadsW = kFewBytes / 16 / kFewThreads, kLoadsH = kFew * D * 2 / 16 / kFewThreads;
    bring_rows<T, D, kLoadsH>(a.H, a.d, 0, a.B, h, PARTS ? a.B : 0);
    bring_rows<T, D, kLoadsW>(a.W, a.d, (long long)blockIdx.x * IT, a.N, w0);
    // what default_rows_kernel does for more positions: these rows are a wave's lanes
    __shared__ float factor_of_all;
    if (wave == 0) {
        const float g = row_weight(a, lane);
        const float top = wave_top(weight_size(g));
        info[lane] = row_info<T>(g, top, a.lse_in[min(position_of(a, lane), a.B - 1)]);
        if (blockIdx.x == 0) a.info[lane] = info[lane];
        if (kOwn) over_top[lane] = g == 0.0f ? 0.0f : g / top;
        target[lane] = lane < dz_rows(a) ? a.targets[position_of(a, lane)] : -1;
        if (lane == 0) factor_of_all = top / kDzScale;
    }
    // dH: 2 x D / 32 blocks of 32 rows x 32 elements, shared by the waves; D = 64 leaves half of them without one
    constexpr int kBlocksH = D / 16 >= kWaves ? D / 16 / kWaves : 1;
    f32x16 dh[kBlocksH];
#pragma unroll
    for (int i = 0; i < kBlocksH; ++i) dh[i] = f32x16{};
    const int h_pos = wave % 2 * 32, h_col = wave / 2 * kBlocksH * 32;         // (a wave's blocks: one half of the rows)

    int turn = 0;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    for (int i = tid; i < kFew * D / 8; i += kFewThreads)      // (a position that adds nothing may hold anything, NaN too)
        if (info[i / (D / 8)].at == __builtin_inff()) reinterpret_cast<uint4*>(h)[i] = uint4{0, 0, 0, 0};
    const float factor = factor_of_all;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x, ++turn) {
        unsigned char* w = turn % 2 ? w1 : w0;
        // every wave's part of the tile has come (below), and every wave is done with the other buffer
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        bring_rows<T, D, kLoadsW>(a.W, a.d, min(tile + gridDim.x, tiles - 1) * IT, a.N, turn % 2 ? w0 : w1);

        // z and dz: blocks of 16 items x 16 rows
        constexpr int kBlocksZ = IT / 16 * 4 / kWaves;
#pragma unroll
        for (int i = 0; i < kBlocksZ; ++i) {
            const int block = wave * kBlocksZ + i, item0 = block / 4 * 16, pos = block % 4 * 16 + lane % 16;
            f32x4_t z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
                z = multiply16<T>(RowsD::along(w, item0 + lane % 16, 4 * k + lane / 16), RowsD::along(h, pos, 4 * k + lane / 16), z);
            const RowInfo r = info[pos];
            const int first = item0 + lane / 16 * 4;
            const long long hit = (long long)target[pos] - (tile * IT + first), left = a.N - (tile * IT + first);
            typedef T T4 __attribute__((ext_vector_type(4)));
            T4 v, u;
            const float over = kOwn ? over_top[pos] : 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float p = exp2_fast(fmaf(z[e], kLog2e, -r.at));
                if (e == hit) p -= kDzScale;
                if (e >= left) p = 0.0f;
                v[e] = (T)(p * r.scale);
                if (PARTS && pos >= a.B) v[e] = (T)fmaf(p, r.scale, -(float)v[e]);
                if (kOwn) {
                    u[e] = (T)(p * over);
                    if (PARTS && pos >= a.B) u[e] = (T)fmaf(p, over, -(float)u[e]);
                }
            }
            *reinterpret_cast<T4*>(dz + RowsI::at(pos, first / 8) + first % 8 * 2) = v;
            if (kOwn) *reinterpret_cast<T4*>(dz_w + RowsI::at(pos, first / 8) + first % 8 * 2) = u;
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");

        if (D / 16 >= kWaves || wave < D / 16) {
#pragma unroll
            for (int k = 0; k < IT / 16; ++k) {
                const s16x8 x = RowsI::along(dz, h_pos + lane % 32, 2 * k + lane / 32);
#pragma unroll
                for (int i = 0; i < kBlocksH; ++i) {
                    const s16x8 xs[1] = {x}, ys[1] = {RowsD::across(w, 16 * k, h_col + 32 * i)};
                    f32x16 c[1][1] = {{dh[i]}};
                    multiply<T, 1, 1>(xs, ys, c);
                    dh[i] = c[0][0];
                }
            }
        }
        // dW: the wave's 32 items x 64 elements
        const int w_item = wave * 2 / (D / 32) * 32, w_col = wave * 2 % (D / 32) * 32;
        f32x16 dw[1][2] = {{f32x16{}, f32x16{}}};
#pragma unroll
        for (int k = 0; k < kFew / 16; ++k) {
            const s16x8 x[1] = {RowsI::across(dz_w, 16 * k, w_item)}, y[2] = {RowsD::across(h, 16 * k, w_col), RowsD::across(h, 16 * k, w_col + 32)};
            multiply<T, 1, 2>(x, y, dw);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // (nobody reads the tile any more: it is the waves' own memory now)
        unsigned char* own = w + wave * 4096;
#pragma unroll
        for (int ni = 0; ni < 2; ++ni)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int row = 8 * (e / 4) + 4 * (lane / 32) + e % 4, byte = (32 * ni + lane % 32) * 2;
                *reinterpret_cast<T*>(own + row * 128 + ((byte / 16) ^ (row % 8)) * 16 + byte % 16) = (T)(dw[0][ni][e] * factor);
            }
        // the wave's part of the next tile has come; what it stores from here on may take until then
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = i * 8 + lane / 8, piece = lane % 8, col = w_col + piece * 8;
            const uint4 v = *reinterpret_cast<const uint4*>(own + row * 128 + ((piece ^ (row % 8)) * 16));
            const long long item = tile * IT + w_item + row;
            if (item < a.N && col < a.d) *reinterpret_cast<uint4*>(static_cast<T*>(a.dW) + (size_t)item * a.d + col) = v;
        }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");                 // (a last load into LDS may be under way)
    if (D / 16 >= kWaves || wave < D / 16) {
#pragma unroll
        for (int i = 0; i < kBlocksH; ++i) {
            const int col = h_col + 32 * i + lane % 32;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int q = h_pos + 8 * (e / 4) + 4 * (lane / 32) + e % 4;
                if (q < dz_rows(a) && col < a.d) a.partial_h[((size_t)blockIdx.x * dz_rows(a) + q) * a.d + col] = dh[i][e];
            }
        }
    }
}

// The slices' shares of dH (a slice's parts follow each other), added: every eighth by one of eight threads, these in their order.  64 positions of 512, 256
// slices: 7.5 us for 34 MB.
template <typename T>
__global__ __launch_bounds__(256) void default_dh_join_kernel(DenseArgs a) {
    __shared__ float part[8][32];
    const size_t n = (size_t)a.B * a.d;
    const int lead = threadIdx.x / 32;
    for (size_t first = (size_t)blockIdx.x * 32; first < n; first += (size_t)gridDim.x * 32) {
        const size_t i = first + threadIdx.x % 32;
        const float factor = a.info[(uint32_t)min(i, n - 1) / (uint32_t)a.d].factor;
        float sum = 0.0f;
        if (i < n) {
#pragma unroll 4
            for (int s = lead; s < a.slices * a.parts; s += 8) sum += a.partial_h[(size_t)s * n + i];
        }
        part[lead][threadIdx.x % 32] = sum;
        __syncthreads();
        if (lead == 0 && i < n) {
#pragma unroll
            for (int w = 1; w < 8; ++w) sum += part[w][threadIdx.x];
            static_cast<T*>(a.dH)[i] = (T)(sum * factor);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------------
// host side, by type of the operands (a translation unit each)

struct DensePlan {
    int loss_items, positions, position_tiles, tiles_each, groups;   // loss: items and positions of a tile of z
    long long item_tiles;
    int parts, piece, pieces, padded, dz_items, dz_positions, dw_items, dw_cols;  // gradient: items and positions of a tile of dz, columns of one of dW
    int rows, cols, rows_tiles, cols_tiles, slices;    // a tile of dH, and how many share its items
    bool few, together;                                // by default_few_kernel; dW and dH in one launch
    size_t info_at, live_at, scaled_at, dz_at, partial_at, bytes;          // its workspace
};

inline int grid_of(long long outer, long long inner) { return (int)(ceil_div(outer, 8) * 8 * inner); }     // see chiplet_order()

constexpr int kSliceItems = 64;                        // a slice of dH's items is a multiple of this
constexpr long long kMostJoinBlocks = 1LL << 20;       // (a launch has fewer than 2^32 threads)

template <typename T> hipError_t dense_loss(const DensePlan& p, const DenseArgs& a, hipStream_t st);
template <typename T> hipError_t dense_backward(const DensePlan& p, DenseArgs a, hipStream_t st);

#ifdef PQ_DENSE_INSTANCE
template <typename T, int POS, int ITEMS>
hipError_t launch_loss(const DensePlan& p, const DenseArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((default_cross_entropy_kernel<T, POS, ITEMS>), dim3(grid_of(p.groups, p.position_tiles)), dim3(ScoresTile<T, POS, ITEMS>::kThreads), 0, st, a);
    return hipGetLastError();
}
template <typename T, int POS, int ITEMS, bool ROWS = false>
hipError_t launch_dz(DenseArgs a, hipStream_t st) {
    a.tiles_m = a.items / ITEMS;
    a.tiles_n = a.padded / POS;
    hipLaunchKernelGGL((default_dz_kernel<T, POS, ITEMS, ROWS>), dim3(grid_of(a.tiles_m, a.tiles_n)), dim3(ScoresTile<T, POS, ITEMS>::kThreads), 0, st, a);
    return hipGetLastError();
}
template <typename T, int COLS, int ITEMS>
hipError_t launch_dw(DenseArgs a, hipStream_t st) {
    a.tiles_m = a.items / ITEMS;
    a.tiles_n = (int)ceil_div(a.d, COLS);
    hipLaunchKernelGGL((default_dw_kernel<T, COLS, ITEMS>), dim3(grid_of(a.tiles_m, a.tiles_n)), dim3(TileW<T, COLS, ITEMS>::kThreads), 0, st, a);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_products(DenseArgs a, hipStream_t st) {
    a.tiles_m = a.items / 64;
    a.tiles_n = (int)ceil_div(a.d, 64);
    a.w_blocks = grid_of(a.tiles_m, a.tiles_n);
    hipLaunchKernelGGL((default_products_kernel<T>), dim3(a.w_blocks + grid_of(a.slices, (long long)a.h_rows * a.h_cols)), dim3(TileW<T, 64, 64>::kThreads), 0, st, a);
    return hipGetLastError();
}
template <typename T, int ROWS, int COLS>
hipError_t launch_dh(const DenseArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((default_dh_kernel<T, ROWS, COLS>), dim3(grid_of(a.slices, (long long)a.h_rows * a.h_cols)), dim3(TileH<T, ROWS, COLS>::kThreads), 0, st, a);
    return hipGetLastError();
}
template <typename T, int ROWS>
hipError_t launch_dh_cols(const DensePlan& p, const DenseArgs& a, hipStream_t st) {
    // (64 positions of narrow 16-bit embeddings are default_few_kernel's)
    if constexpr (ROWS == 64 && sizeof(T) == 2) return launch_dh<T, ROWS, 256>(a, st);
    else return p.cols == 256 ? launch_dh<T, ROWS, 256>(a, st) : p.cols == 128 ? launch_dh<T, ROWS, 128>(a, st) : launch_dh<T, ROWS, 64>(a, st);
}

template <typename T>
hipError_t launch_few_loss(const DensePlan& p, const DenseArgs& a, hipStream_t st) {
    const dim3 grid(p.groups), threads(kFewThreads);
    if (a.d > 256) hipLaunchKernelGGL((default_few_loss_kernel<T, 512>), grid, threads, 0, st, a);
    else if (a.d > 128) hipLaunchKernelGGL((default_few_loss_kernel<T, 256>), grid, threads, 0, st, a);
    else if (a.d > 64) hipLaunchKernelGGL((default_few_loss_kernel<T, 128>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((default_few_loss_kernel<T, 64>), grid, threads, 0, st, a);
    return hipGetLastError();
}
template <typename T, bool PARTS>
hipError_t launch_few_of(const DensePlan& p, const DenseArgs& a, hipStream_t st) {
    const dim3 grid(p.slices), threads(kFewThreads);
    if (a.d > 256) hipLaunchKernelGGL((default_few_kernel<T, 512, PARTS>), grid, threads, 0, st, a);
    else if (a.d > 128) hipLaunchKernelGGL((default_few_kernel<T, 256, PARTS>), grid, threads, 0, st, a);
    else if (a.d > 64) hipLaunchKernelGGL((default_few_kernel<T, 128, PARTS>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((default_few_kernel<T, 64, PARTS>), grid, threads, 0, st, a);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_few(const DensePlan& p, const DenseArgs& a, hipStream_t st) { return a.parts > 1 ? launch_few_of<T, true>(p, a, st) : launch_few_of<T, false>(p, a, st); }

template <typename T>
hipError_t dense_loss(const DensePlan& p, const DenseArgs& a, hipStream_t st) {
    hipError_t e;
    if constexpr (sizeof(T) == 2) e = p.few ? launch_few_loss<T>(p, a, st) : hipSuccess;
    if (sizeof(T) != 2 || !p.few)
        e = p.loss_items == 64 ? launch_loss<T, 64, 64>(p, a, st) : p.positions == 256 ? launch_loss<T, 256, 256>(p, a, st)
            : p.positions == 128 ? launch_loss<T, 128, 256>(p, a, st) : launch_loss<T, 64, 256>(p, a, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((default_cross_entropy_join_kernel<T>), dim3(a.B), dim3(kWave), 0, st, a);
    return hipGetLastError();
}

template <typename T>
hipError_t dense_backward(const DensePlan& p, DenseArgs a, hipStream_t st) {
    hipError_t e = hipSuccess;
    if constexpr (sizeof(T) == 2) {
        if (p.few) e = launch_few<T>(p, a, st);
    }
    const void* queries = a.H;
    const bool own_rows = a.B <= 64 && !kOwnPowers<T>;         // (then dz's rows are those of one tile)
    if (!p.few && !own_rows) {
        const long long row_blocks = ceil_div((long long)a.B * a.parts * a.d * (long long)sizeof(T), 16 * 1024);
        const dim3 grid((unsigned)(row_blocks < kCUs ? row_blocks : kCUs));
        hipLaunchKernelGGL((default_rows_kernel<T>), grid, dim3(1024), 0, st, a);
        e = hipGetLastError();
        queries = a.live;
        if constexpr (kOwnPowers<T>) {
            if (e == hipSuccess) {
                hipLaunchKernelGGL((scale_rows_kernel<T>), grid, dim3(1024), 0, st, a);
                e = hipGetLastError();
            }
        }
    }
    for (int i = 0; !p.few && i < p.pieces && e == hipSuccess; ++i) {
        a.first_item = (long long)i * p.piece;
        const long long left = a.N - a.first_item;
        a.items = (int)round_up((size_t)(left < p.piece ? left : p.piece), kItems);
        a.more = i > 0;
        a.H = queries;
        if constexpr (!kOwnPowers<T>) {
            if (own_rows) e = p.dz_items == 64 ? launch_dz<T, 64, 64, true>(a, st) : launch_dz<T, 64, 256, true>(a, st);
        }
        if (!own_rows) e = p.dz_items == 64 ? launch_dz<T, 64, 64>(a, st) : p.dz_positions == 256 ? launch_dz<T, 256, 256>(a, st)
            : p.dz_positions == 128 ? launch_dz<T, 128, 256>(a, st) : launch_dz<T, 64, 256>(a, st);
        if (e != hipSuccess) break;
        a.H = kOwnPowers<T> ? a.scaled : a.live;
        a.h_rows = p.rows_tiles;
        a.h_cols = p.cols_tiles;
        a.slice_items = (int)round_up((size_t)ceil_div(a.items, p.slices), kSliceItems);
        if (p.together) {
            e = launch_products<T>(a, st);
            continue;
        }
        e = p.dw_items == 64 ? launch_dw<T, 64, 64>(a, st) : p.dw_cols == 256 ? launch_dw<T, 256, 256>(a, st)
            : p.dw_cols == 128 ? launch_dw<T, 128, 256>(a, st) : launch_dw<T, 64, 256>(a, st);
        if (e != hipSuccess) break;
        e = p.rows == 256 ? launch_dh_cols<T, 256>(p, a, st) : p.rows == 128 ? launch_dh_cols<T, 128>(p, a, st) : launch_dh_cols<T, 64>(p, a, st);
    }
    if (e != hipSuccess) return e;
    const long long join_blocks = ceil_div((long long)a.B * a.d, 32);
    hipLaunchKernelGGL((default_dh_join_kernel<T>), dim3((unsigned)(join_blocks < kMostJoinBlocks ? join_blocks : kMostJoinBlocks)), dim3(256), 0, st, a);
    return hipGetLastError();
}

template hipError_t dense_loss<PQ_DENSE_INSTANCE>(const DensePlan&, const DenseArgs&, hipStream_t);
template hipError_t dense_backward<PQ_DENSE_INSTANCE>(const DensePlan&, DenseArgs, hipStream_t);
#endif

}  // namespace head
}  // namespace pqk
