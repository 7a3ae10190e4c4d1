// pq_default_cross_entropy and its gradient: checks, plans and entry points (the kernels: default_cross_entropy.hpp).
#include "default_cross_entropy.hpp"

namespace pqk {
namespace head {
namespace {

// Bytes of dz's buffer.  Fewer, longer launches gain more than a buffer of the last-level cache's size (gradient, us, 256 MB and
// 1 GB of bfloat16: 1.28M items of 128, 256 positions 756 and 660; of 512, 1024 positions 4550 and 4410; 600,000 of 256, 512
// positions 794 and 708; float32, 512 MB and 1 GB, 1 to 4 %), but for short rows, whose products wait for dz alone (bfloat16,
// 1.28M of 64, 512 positions 943 and 995).
constexpr long long kDzBytes = 1LL << 30, kDzBytesShort = 1LL << 28;
constexpr long long kMaxPiece = 1LL << 22;
constexpr long long kMostLossBlocks = 64 * kCUs;

// What a tile of 256 rows and `cols` columns takes a compute unit next to one of 256 x 256 that keeps the matrix cores as busy
// as can be (the smaller ones' rates: 203 of 208 TFLOP/s and about 165 in float32; 880 of 1040 and about 600 in 16 bits).
// Two workgroups of a smaller tile share a compute unit, but one alone has nearly all of it: what counts is how many a
// compute unit gets.
double tile_cost(int cols, int size) {
    const bool f32 = size == 4;
    return cols == 256 ? 1.0 : cols == 128 ? 0.5 / (f32 ? 0.97 : 0.86) : 0.25 / (f32 ? 0.8 : 0.6);
}
constexpr double kTileStart = 0.1;                     // what a workgroup takes besides its products

int size_of(int type) { return type == PQ_FLOAT32 ? 4 : type == PQ_BFLOAT16 || type == PQ_FLOAT16 ? 2 : 0; }

DensePlan plan_dense(long long N, int B, int d, int type) {
    DensePlan p;
    const int size = size_of(type);
    // Tiles of 64 x 64 where all of them run at once (loss and gradient, us: 10,000 items of 64 float32, 50 positions 42 with tiles
    // of 256 x 64, 34 so; 5000 of 512, one position 81 and 54; 8000 of 512, 128 positions 98 and 73), and for dz somewhat longer
    // (gradient: 5000 of 128, 1000 positions 57 and 49; 10,000 of 512, 500 positions 152 and 143; 8000 of 512, 900 positions 179 and
    // 195, bfloat16 66 and 66).  The loss's larger tiles fold several tiles of items before they leave a sum.
    auto small_tiles = [](long long items, long long width, int rounds) { return ceil_div(items, 64) * ceil_div(width, 64) <= rounds * kCUs; };
    p.loss_items = small_tiles(N, B, 2) ? 64 : kItems;
    p.item_tiles = ceil_div(N, p.loss_items);
    // loss: the tiles of positions, and how many tiles of items a workgroup takes, whose rounds over the chip take least
    double best = 1e300;
    for (int tile : {256, 128, 64}) {
        // (of short rows in 16 bits a tile's exponentials take longer than its products: two workgroups of 128 positions on a compute
        // unit do one while the other does the other; 300,000 items of 64, 2048 positions 235 and 201 us, of 128, 1024 positions
        // 143 and 136, of 256 the same)
        if (tile == 256 && size == 2 && d <= 128) continue;
        for (int each = 1; each <= 64; each *= 2) {
            const long long position_tiles = ceil_div(B, tile), groups = ceil_div(p.item_tiles, each);
            const double cost = (double)ceil_div(groups * position_tiles, kCUs) * (each * tile_cost(tile, size) + kTileStart);
            if (cost < best * 0.99) {
                best = cost;
                p.positions = tile; p.position_tiles = (int)position_tiles; p.tiles_each = each; p.groups = (int)groups;
            }
        }
    }
    // (a workgroup more is nothing to gain where there are many to a compute unit, but a sum more to keep: long catalogues of many
    // positions would launch 2^32 threads, which HIP refuses, and ask for gigabytes of sums)
    while ((long long)p.groups * p.position_tiles > kMostLossBlocks) {
        p.tiles_each *= 2;
        p.groups = (int)ceil_div(p.item_tiles, p.tiles_each);
    }
    if (p.loss_items == 64) {
        p.positions = 64; p.position_tiles = (int)ceil_div(B, 64); p.tiles_each = 1; p.groups = (int)p.item_tiles;
    }
    // gradient: pieces of the items, in balance
    p.parts = size == 2 && B <= kTwoParts ? 2 : 1;
    const int small = B <= 64 ? 64 : 128;              // (positions are padded to a multiple of this or of 256)
    long long piece = (size == 2 && d <= 64 ? kDzBytesShort : kDzBytes) / size / (long long)round_up(B, small);
    if (piece < 2048) piece = 2048;
    if (piece > kMaxPiece) piece = kMaxPiece;
    p.pieces = (int)ceil_div(N, piece);
    p.piece = (int)round_up((size_t)ceil_div(N, p.pieces), kItems);
    p.pieces = (int)ceil_div(N, p.piece);
    const long long tiles = p.piece / kItems;
    best = 1e300;
    for (int tile : {256, 128, 64}) {
        const double cost = (double)ceil_div(tiles * ceil_div(B, tile), kCUs) * (tile_cost(tile, size) + kTileStart);
        if (cost < best * 0.99) { best = cost; p.dz_positions = tile; }
    }
    p.dz_items = small_tiles(p.piece, B, 5) ? 64 : kItems;
    if (p.dz_items == 64) p.dz_positions = 64;
    p.padded = (int)round_up(B, p.dz_positions);
    best = 1e300;
    for (int cols : {256, 128, 64}) {
        const double cost = (double)ceil_div(tiles * ceil_div(d, cols), kCUs) * (tile_cost(cols, size) * p.padded / 512.0 + kTileStart);
        if (cost < best * 0.99) { best = cost; p.dw_cols = cols; }
    }
    p.dw_items = small_tiles(p.piece, d, 2) ? 64 : kItems;
    // dH: as many slices of the items as fill the chip once
    // dW and dH in one launch, by tiles of 64 x 64, until there are enough of these that larger ones gain more than a launch takes
    // (gradient, us, apart and together; float32: 5000 items of 512, one position 37 and 30; 10,000 of 256, 200 positions 68 and 51;
    // 10,000 of 512, 300 positions 111 and 106; 60,000 of 128, 300 positions 144 and 144; 500,000 of 64, 33 positions 152 and 167;
    // bfloat16: 10,000 of 256, 200 positions 40 and 28; 34,742 of 512, 128 positions 69 and 52; 5000 of 512, 1500 positions 98 and 102).
    p.together = ceil_div(B, 64) * ceil_div(p.piece, 64) * ceil_div(d, 64) <= (size == 4 ? 24 : 48) * kCUs;
    p.rows = p.together ? 64 : B > 128 ? 256 : B > 64 ? 128 : 64;
    p.cols = p.together ? 64 : d > 128 ? 256 : d > 64 ? 128 : 64;
    p.rows_tiles = (int)ceil_div(B, p.rows);
    p.cols_tiles = (int)ceil_div(d, p.cols);
    const bool big = p.rows == 256 && p.cols == 256;
    long long slices = (big ? 1LL : 2LL) * kCUs / ((long long)p.rows_tiles * p.cols_tiles);
    const long long most = p.piece / kSliceItems;
    p.slices = (int)(slices < 1 ? 1 : slices > most ? most : slices);
    p.few = size == 2 && B <= kFew && d <= 512;
    if (p.few) {                                       // a workgroup per compute unit; dz stays in LDS
        const long long few_tiles = ceil_div(N, kFewBytes / 2 / (d > 256 ? 512 : d > 128 ? 256 : d > 64 ? 128 : 64));
        p.slices = p.groups = (int)(few_tiles < kCUs ? few_tiles : kCUs);
        p.padded = kFew;
        p.piece = 0;
    }
    const size_t query_bytes = (size_t)B * p.parts * d * size;
    p.info_at = 256 + kCUs * sizeof(int);              // (dW's factor, the blocks' powers)
    p.live_at = round_up(p.info_at + (size_t)p.padded * sizeof(RowInfo), 256);
    p.scaled_at = round_up(p.live_at + (p.few ? 0 : query_bytes), 256);
    p.dz_at = round_up(p.scaled_at + (p.few || type != PQ_FLOAT16 ? 0 : query_bytes), 256);
    p.partial_at = round_up(p.dz_at + (size_t)p.padded * p.piece * size, 256);
    p.bytes = round_up(p.partial_at + (size_t)p.slices * B * p.parts * d * sizeof(float), 256);
    return p;
}

int check_dense(long long N, int B, int d, int type) {
    if (N < 1 || B < 1 || d < 1 || N >= 2147483648LL || size_of(type) == 0) return PQ_ERR_SHAPE;
    if (B > PQ_MAX_B || d > 16384 || d % (16 / size_of(type)) != 0) return PQ_ERR_UNSUPPORTED;
    return PQ_OK;
}

size_t loss_bytes(const DensePlan& p, int B) { return round_up((size_t)p.groups * B * sizeof(float2), 16); }

}  // namespace
}  // namespace head
}  // namespace pqk

using namespace pqk::head;

extern "C" {

size_t pq_default_cross_entropy_workspace_bytes(long long N, int B, int d, int type) {
    return check_dense(N, B, d, type) == PQ_OK ? loss_bytes(plan_dense(N, B, d, type), B) : 0;
}

int pq_default_cross_entropy(const void* W, const void* queries, const int* targets, long long N, int B, int d, int type, float* loss,
                             float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!W || !queries || !targets || !loss || !lse || !workspace) return PQ_ERR_NULL;
    const int rc = check_dense(N, B, d, type);
    if (rc != PQ_OK) return rc;
    if ((((uintptr_t)W | (uintptr_t)queries | (uintptr_t)workspace) & 15) || (((uintptr_t)targets | (uintptr_t)loss | (uintptr_t)lse) & 3)) return PQ_ERR_ALIGN;
    const DensePlan p = plan_dense(N, B, d, type);
    if (workspace_bytes < loss_bytes(p, B)) return PQ_ERR_WORKSPACE;
    DenseArgs a{};
    a.W = W; a.H = queries; a.targets = targets; a.N = N; a.B = B; a.d = d;
    a.item_tiles = p.item_tiles; a.tiles_each = p.tiles_each; a.groups = p.groups; a.position_tiles = p.position_tiles;
    a.partial = static_cast<float2*>(workspace); a.loss = loss; a.lse = lse;
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (type == PQ_FLOAT32) e = dense_loss<float>(p, a, st);
    else if (type == PQ_BFLOAT16) e = dense_loss<__bf16>(p, a, st);
    else e = dense_loss<_Float16>(p, a, st);
    return pqk::record_hip_error(e);
}

size_t pq_default_cross_entropy_backward_workspace_bytes(long long N, int B, int d, int type) {
    return check_dense(N, B, d, type) == PQ_OK ? plan_dense(N, B, d, type).bytes : 0;
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
    const DensePlan p = plan_dense(N, B, d, type);
    if (workspace_bytes < p.bytes) return PQ_ERR_WORKSPACE;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    DenseArgs a{};
    a.W = W; a.H = queries; a.targets = targets; a.N = N; a.B = B; a.d = d;
    a.lse_in = lse; a.grad = grad_loss; a.dH = dqueries; a.dW = dW;
    a.factor = reinterpret_cast<float*>(ws);
    a.block_powers = reinterpret_cast<int*>(ws + 256);
    a.info = reinterpret_cast<RowInfo*>(ws + p.info_at);
    a.live = ws + p.live_at;
    a.scaled = ws + p.scaled_at;
    a.dz = ws + p.dz_at;
    a.partial_h = reinterpret_cast<float*>(ws + p.partial_at);
    a.parts = p.parts; a.piece = p.piece; a.padded = p.padded; a.slices = p.slices;
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (type == PQ_FLOAT32) e = dense_backward<float>(p, a, st);
    else if (type == PQ_BFLOAT16) e = dense_backward<__bf16>(p, a, st);
    else e = dense_backward<_Float16>(p, a, st);
    return pqk::record_hip_error(e);
}

}  // extern "C"
