// The default scorer's scores from four-bit item embeddings (pq_default_scores_q4), and how these are made (pq_quantise_items).
//
//   r_qi = sum_g scale[i][g] * sum_{e in group g} (n[i][e] - 8) * phi[q][e]        n in 0..15
#include "pqtopk.h"
#include "head_common.hpp"

namespace pqk {
namespace head {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr int kStep = 128;                           // elements of an embedding per step: 64 bytes of a row, 16 for a lane
constexpr int kTileItems = 16, kTiles = 2;           // items of a matrix instruction; instructions side by side

struct Q4Args {
    const uint8_t* packed;      // [N][d / 2]
    const uint16_t* scales;     // [N][d / group], bfloat16
    const float* queries;       // [B][d]
    float* scores;              // [B][ld]
    long long N, ld, item_tiles;
    int B, d, steps;            // steps = d / 128, rounded up
    int held;                   // tile pairs whose scores a wave holds back
};

// A query element as a whole number of 31 bits, in four signed bytes: v = d0 + 2^8 d1 + 2^16 d2 + 2^24 d3.
__device__ __forceinline__ uint32_t four_digits(float x, int shift) {
    const int v = __float2int_rn(ldexpf(x, shift));
    // adding 128 to each byte in turn carries what a byte beyond 127 owes the next one
    return ((uint32_t)v + 0x00808080u) ^ 0x00808080u;
}

// Scores on the integer matrix cores: both operands are whole numbers and a digit's sums are exact (below 2^21).  Rounded are
// the query (to 2^-31 of a power of two above its largest element: less than float32 there), a group's sum, joined from its
// four digits in float32, and the float32 sum over groups.
// The instruction's 16 rows are four queries' four digits, its 16 columns items: a lane finishes one score, all its digits
// at hand, with its item's scale.
// Bound by the stream of nibbles, which comes in 16 bytes a lane, 64 neighbouring bytes of sixteen rows an instruction (with
// 8 bytes a lane the same stream reached 4.4 TB/s instead of 5.9).  Those 64 bytes are 128 elements: two groups of 64, four of
// 32.  Each group's sums are taken from all lanes' weights with the other groups' digits zeroed: the matrix cores have the
// time, as four queries ask for 2 PARTS instructions of 16 cycles per 1 KB of weights.
// Scores are held back in LDS and leave a wave's tiles at a time: stores between the loads cost the stream more than their
// bytes (1.3 GB read by 128 bytes stored per 8 KB: 207 us without stores, 262 with, 227 held back).
// Registers leave room for two workgroups where one set of queries and its groups let them, but for groups of 32 with scales
// of odd rows: held to 128 registers those spill (1.28M items of 96 elements, one query: 49.4 us, with one workgroup 45.4).
// GROUP: weights that share a scale; SETS: sets of four queries a pass over the weights serves; WHOLE: d is a multiple of 128.
template <int SETS, int GROUP, bool WHOLE>
__global__ __launch_bounds__(kThreads, SETS * (kStep / GROUP) <= 4 && (GROUP > 32 || WHOLE) ? 4 : 2) void default_scores_q4_kernel(Q4Args a) {
    constexpr int PARTS = kStep / GROUP;                       // groups a step
    constexpr int kAhead = 4;                                  // steps whose weights are on their way
    constexpr bool kHold = SETS <= 2;
    extern __shared__ __align__(16) unsigned char smem[];
    i32x4* digits = reinterpret_cast<i32x4*>(smem);            // [step][half][set][lane]: as the matrix instruction takes them
    float* factor = reinterpret_cast<float*>(digits + (size_t)a.steps * 2 * SETS * kWave);       // [query]
    int* shift = reinterpret_cast<int*>(factor + SETS * 4);
    float* held = reinterpret_cast<float*>(shift + SETS * 4);                                    // [wave][tile pair][query][32 items]
    const int groups = a.d / GROUP;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int q0 = blockIdx.y * SETS * 4;

    const int col = lane % 16, h = lane / 16;
    const size_t row_bytes = (size_t)a.d / 2;
    const long long last_item = a.N - 1, waves = (long long)gridDim.x * kWaves;
    // A wave's work is one sequence of steps, those of a tile pair and then of the next one.  The weights of kAhead steps are
    // always on their way: waves that all waited for a round of loads would leave the memory idle while they compute.
    typedef uint16_t Scales __attribute__((ext_vector_type(PARTS)));
    const long long tiles_end = (a.item_tiles + kTiles - 1) / kTiles, first_tile = (long long)blockIdx.x * kWaves + wave;
    uint4 ring_w[kAhead][kTiles];
    Scales ring_s[kAhead][kTiles];
    long long load_tile = first_tile;
    int load_step = 0;
    auto load = [&](int slot) {
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            const long long item = min((load_tile * kTiles + u) * kTileItems + col, last_item);
            // past the row's end the digits are zero: any weights will do
            ring_w[slot][u] = *reinterpret_cast<const uint4*>(a.packed + (size_t)item * row_bytes + min(load_step * (kStep / 2) + 16 * h, (int)row_bytes - 16));
            // every fourth step brings the scales of four, a step for each of the item's lanes
            if (load_step % 4 == 0) {
                const uint16_t* scale = a.scales + (size_t)item * groups;
                const int step = min(load_step + h, a.steps - 1);
                if constexpr (WHOLE) ring_s[slot][u] = *reinterpret_cast<const Scales*>(scale + step * PARTS);
                else {
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) ring_s[slot][u][p] = scale[min(step * PARTS + p, groups - 1)];
                }
            }
        }
        if (++load_step == a.steps) { load_step = 0; load_tile += waves; }
    };
    if (first_tile < tiles_end) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(i);              // (while the queries are laid out)
    }

    // factors: one wave per query in turn
    for (int s = wave; s < SETS * 4; s += kWaves) {
        float top = 0.0f;
        bool odd = false;
        if (q0 + s < a.B)
            for (int e = lane; e < a.d; e += kWave) {
                const float x = a.queries[(size_t)(q0 + s) * a.d + e];
                top = fmaxf(top, fabsf(x));
                odd |= !(fabsf(x) < __builtin_inff());
            }
#pragma unroll
        for (int x = 1; x < kWave; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
        const bool any_odd = __any(odd);
        if (lane == 0) {
            int e = 0;
            if (top > 0.0f && !any_odd) (void)frexpf(top, &e);           // top < 2^e
            // digits are of x 2^(30 - e); a nibble stands for 16 (n - 8) below.  A query of tiny numbers goes as far as float32 does.
            shift[s] = any_odd ? 0 : e > -92 ? 30 - e : 122;
            factor[s] = any_odd ? __builtin_nanf("") : ldexpf(1.0f, e > -92 ? e - 34 : -126);
        }
    }
    __syncthreads();
    // row r of the instruction is digit r % 4 of query r / 4; a lane's 16 bytes are elements 32 (lane / 16) + 16 half .. + 15 of
    // the step, the even and odd ones of each eight apart, as the nibbles of a word come out
    for (int i = threadIdx.x; i < a.steps * 2 * SETS * kWave; i += kThreads) {
        const int l = i % kWave, set = i / kWave % SETS, half = i / kWave / SETS % 2, step = i / kWave / SETS / 2;
        const int row = l % 16, q = set * 4 + row / 4, first = step * kStep + 32 * (l / 16) + 16 * half;
        uint32_t w[4] = {0, 0, 0, 0};
        if (q0 + q < a.B && first < a.d && factor[q] == factor[q]) {     // (d is a multiple of 32: sixteen elements are there or not)
            const float* phi = a.queries + (size_t)(q0 + q) * a.d + first;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t byte = (four_digits(phi[e], shift[q]) >> (8 * (row % 4))) & 255u;
                w[e / 8 * 2 + e % 2] |= byte << (8 * (e % 8 / 2));
            }
        }
        digits[i] = i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
    }
    __syncthreads();

    int mine[PARTS];                                           // all ones where the lane's elements belong to the step's group p
#pragma unroll
    for (int p = 0; p < PARTS; ++p) mine[p] = h * PARTS / 4 == p ? -1 : 0;
    float sum[kTiles][SETS];
    auto clear = [&] {
#pragma unroll
        for (int u = 0; u < kTiles; ++u)
#pragma unroll
            for (int s = 0; s < SETS; ++s) sum[u][s] = 0.0f;
    };
    clear();
    long long tile = first_tile;
    int step = 0, pairs = 0;
    Scales four_steps[kTiles] = {};
    const int queries = min(SETS * 4, a.B - q0);
    held += (size_t)wave * a.held * queries * 32;
    auto release = [&](long long last_tile) {                  // the held scores, the last of them of last_tile
        wave_reads_after_writes();
        for (int r = lane / 32; r < pairs * queries; r += 2) {
            const int pair = r / queries, q = r - pair * queries;
            const long long item = (last_tile - (long long)(pairs - 1 - pair) * waves) * kTiles * kTileItems + lane % 32;
            if (item < a.N) a.scores[(size_t)(q0 + q) * a.ld + item] = held[r * 32 + lane % 32];
        }
        wave_reads_after_writes();
        pairs = 0;
    };
    // (whole rounds of the ring: steps past the wave's last tile are of items past the last one and leave nothing)
    const int rounds = first_tile < tiles_end ? (int)(((tiles_end - 1 - first_tile) / waves + 1) * a.steps + kAhead - 1) / kAhead : 0;
    for (int round = 0; round < rounds; ++round) {
#pragma unroll
        for (int slot = 0; slot < kAhead; ++slot) {
            __builtin_amdgcn_sched_barrier(0);                 // (steps one after the other: their accumulators share registers)
            i32x4 n[2][kTiles];
            float scale[kTiles][PARTS];
#pragma unroll
            for (int u = 0; u < kTiles; ++u) {
                // a nibble's two's complement of n - 8 in the high half of a byte: 16 (n - 8)
                const uint4 w = ring_w[slot][u];
                const uint32_t v[4] = {w.x ^ 0x88888888u, w.y ^ 0x88888888u, w.z ^ 0x88888888u, w.w ^ 0x88888888u};
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    n[half][u] = i32x4{(int)(v[2 * half] << 4 & 0xF0F0F0F0u), (int)(v[2 * half] & 0xF0F0F0F0u),
                                       (int)(v[2 * half + 1] << 4 & 0xF0F0F0F0u), (int)(v[2 * half + 1] & 0xF0F0F0F0u)};
                if (step % 4 == 0) four_steps[u] = ring_s[slot][u];
                uint32_t words[(PARTS + 1) / 2] = {};
                __builtin_memcpy(words, &four_steps[u], sizeof(Scales));
#pragma unroll
                for (int p = 0; p < PARTS; p += 2) {
                    const uint32_t word = (uint32_t)__shfl((int)words[p / 2], col + 16 * (step % 4));
                    scale[u][p] = __uint_as_float(word << 16);
                    if (p + 1 < PARTS) scale[u][p + 1] = __uint_as_float(word & 0xFFFF0000u);
                }
            }
            load(slot);
#pragma unroll
            for (int s = 0; s < SETS; ++s) {
                const i32x4 x = digits[((size_t)step * 2 * SETS + s) * kWave + lane], y = digits[((size_t)(step * 2 + 1) * SETS + s) * kWave + lane];
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    const i32x4 xp = PARTS == 1 ? x : x & mine[p], yp = PARTS == 1 ? y : y & mine[p];
                    i32x4 acc[kTiles];
#pragma unroll
                    for (int u = 0; u < kTiles; ++u) acc[u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(xp, n[0][u], i32x4{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                    for (int u = 0; u < kTiles; ++u) acc[u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(yp, n[1][u], acc[u], 0, 0, 0);
#pragma unroll
                    for (int u = 0; u < kTiles; ++u) {
                        const float high = (float)((acc[u][3] << 8) + acc[u][2]), low = (float)((acc[u][1] << 8) + acc[u][0]);
                        const float z = fmaf(high, 65536.0f, low);
                        sum[u][s] = fmaf(z, scale[u][p], sum[u][s]);
                    }
                }
            }
            if (++step == a.steps) {
#pragma unroll
                for (int u = 0; u < kTiles; ++u) {
                    const long long item = (tile * kTiles + u) * kTileItems + col;
#pragma unroll
                    for (int s = 0; s < SETS; ++s) {
                        const int q = s * 4 + h;
                        const float z = sum[u][s] * factor[q];
                        if (kHold) { if (q < queries) held[(pairs * queries + q) * 32 + u * kTileItems + col] = z; }
                        else if (item < a.N && q < queries) a.scores[(size_t)(q0 + q) * a.ld + item] = z;
                    }
                }
                if (kHold && ++pairs == a.held) release(tile);
                clear();
                step = 0;
                tile += waves;
            }
        }
    }
    if (kHold && pairs > 0) release(tile - waves);
}

// Eight elements a lane; the lanes of a group share its largest absolute value.  A stream of 4 N d bytes in.
__global__ __launch_bounds__(256) void quantise_items_kernel(const float* W, long long pieces, int lanes_per_group, uint32_t* packed, uint16_t* scales) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (long long)gridDim.x * 256) {
        const float4 x = reinterpret_cast<const float4*>(W)[2 * i], y = reinterpret_cast<const float4*>(W)[2 * i + 1];
        const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        uint32_t top = 0;                                      // (magnitudes in the order of their bits: NaN above all)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
        // (a group's lanes are neighbours of one wave and run this together: the pieces are a multiple of a group's)
        for (int s = 1; s < lanes_per_group; s *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, s));
        // the scale is rounded to bfloat16 (nearest even) first, the weights then to multiples of what is kept; infinities and
        // NaN leave a scale of NaN
        const uint32_t bits = __float_as_uint(__uint_as_float(top) / 7.0f);
        const uint32_t kept = top >= 0x7F800000u ? 0x7FC0u : (bits + 0x7FFFu + (bits >> 16 & 1u)) >> 16;
        const float scale = __uint_as_float(kept << 16);
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float n = scale > 0.0f ? fminf(fmaxf(rintf(v[e] / scale), -8.0f), 7.0f) : 0.0f;
            word |= (uint32_t)((int)n + 8) << (4 * e);
        }
        packed[i] = word;
        if (i % lanes_per_group == 0) scales[i / lanes_per_group] = (uint16_t)kept;
    }
}

int check_q4(long long N, int B, int d, int group) {
    if (N < 1 || B < 1 || d < 1 || N >= 2147483648LL || (group != 32 && group != 64 && group != 128) || d % group != 0) return PQ_ERR_SHAPE;
    if (B > PQ_MAX_B || d > 16384) return PQ_ERR_UNSUPPORTED;
    return PQ_OK;
}

// digits, factors and shifts; then the scores that are held back
size_t q4_lds(int sets, int d) { return (size_t)ceil_div(d, kStep) * 2 * sets * kWave * 16 + (size_t)sets * 4 * 8; }
size_t held_bytes(int queries) { return (size_t)kWaves * queries * 32 * sizeof(float); }          // a tile pair of every wave

template <int SETS, int GROUP, bool WHOLE>
hipError_t go_q4(Q4Args a, hipStream_t st) {
    const size_t fixed = q4_lds(SETS, a.d), pair = SETS <= 2 ? held_bytes(a.B < SETS * 4 ? a.B : SETS * 4) : 16;
    a.item_tiles = ceil_div(a.N, kTileItems);
    const int query_groups = (int)ceil_div(a.B, SETS * 4), per_cu = fixed + pair > kMaxLds / 2 ? 1 : 2;
    const long long pairs = ceil_div(a.item_tiles, kTiles);
    long long blocks = ceil_div(pairs, kWaves);
    if (blocks > (long long)per_cu * kCUs) blocks = (long long)per_cu * kCUs;
    const long long each = ceil_div(pairs, blocks * kWaves), room = (long long)((kMaxLds / per_cu - fixed) / pair);
    a.held = (int)(each < room ? each : room);
    const size_t lds = fixed + a.held * pair;
    hipError_t e = allow_lds(default_scores_q4_kernel<SETS, GROUP, WHOLE>, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((default_scores_q4_kernel<SETS, GROUP, WHOLE>), dim3((unsigned)blocks, query_groups), dim3(kThreads), lds, st, a);
    return hipGetLastError();
}

template <int GROUP, bool WHOLE>
hipError_t go_q4_sets(const Q4Args& a, hipStream_t st) {
    // as many queries a pass over the weights as there are, up to 32 and what LDS holds of their digits
    int sets = a.B <= 4 ? 1 : a.B <= 8 ? 2 : a.B <= 16 ? 4 : 8;
    while (sets > 1 && q4_lds(sets, a.d) + held_bytes(sets * 4) > kMaxLds) sets /= 2;
    return sets == 8 ? go_q4<8, GROUP, WHOLE>(a, st) : sets == 4 ? go_q4<4, GROUP, WHOLE>(a, st) : sets == 2 ? go_q4<2, GROUP, WHOLE>(a, st) : go_q4<1, GROUP, WHOLE>(a, st);
}

template <int GROUP>
hipError_t go_q4_group(const Q4Args& a, hipStream_t st) {
    if (GROUP == kStep || (a.d % kStep == 0 && ((uintptr_t)a.scales & 7) == 0)) return go_q4_sets<GROUP, true>(a, st);
    return go_q4_sets<GROUP, GROUP == kStep>(a, st);
}

}  // namespace
}  // namespace head
}  // namespace pqk

using namespace pqk::head;

extern "C" {

int pq_quantise_items(const float* W, long long N, int d, int group, uint8_t* packed, uint16_t* scales, void* stream) {
    if (!W || !packed || !scales) return PQ_ERR_NULL;
    const int rc = check_q4(N, 1, d, group);
    if (rc != PQ_OK) return rc;
    if (((uintptr_t)W & 15) || ((uintptr_t)packed & 15) || ((uintptr_t)scales & 1)) return PQ_ERR_ALIGN;
    const long long pieces = N * d / 8;
    long long blocks = ceil_div(pieces, 256);
    if (blocks > 32 * kCUs) blocks = 32 * kCUs;
    hipLaunchKernelGGL(quantise_items_kernel, dim3((unsigned)blocks), dim3(256), 0, static_cast<hipStream_t>(stream), W, pieces, group / 8,
                       reinterpret_cast<uint32_t*>(packed), scales);
    return pqk::record_hip_error(hipGetLastError());
}

int pq_default_scores_q4(const uint8_t* packed, const uint16_t* scales, const float* queries, long long N, int B, int d, int group,
                         float* scores, long long ld, void* stream) {
    if (!packed || !scales || !queries || !scores) return PQ_ERR_NULL;
    const int rc = check_q4(N, B, d, group);
    if (rc != PQ_OK) return rc;
    if (ld < N) return PQ_ERR_SHAPE;
    if (q4_lds(1, d) + held_bytes(4) > kMaxLds) return PQ_ERR_UNSUPPORTED;
    if (((uintptr_t)packed & 15) || ((uintptr_t)scales & 1) || (((uintptr_t)queries | (uintptr_t)scores) & 3)) return PQ_ERR_ALIGN;
    const Q4Args a{packed, scales, queries, scores, N, ld, 0, B, d, (int)ceil_div(d, kStep)};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return pqk::record_hip_error(group == 32 ? go_q4_group<32>(a, st) : group == 64 ? go_q4_group<64>(a, st) : go_q4_group<128>(a, st));
}

}  // extern "C"
