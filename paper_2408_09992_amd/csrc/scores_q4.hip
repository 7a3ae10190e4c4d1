// The default scorer's scores from four-bit item embeddings (pq_default_scores_q4), and how these are made (pq_quantise_items).
//
//   r_qi = sum_g scale[i][g] * sum_{e in group g} (n[i][e] - 8) * phi[q][e]        n in 0..15
#include "pqtopk.h"
#include "head_common.hpp"

namespace pqk {
namespace head {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr int kStep = 128, kQuarters = 4;            // elements of a row per step: 64 bytes, a quarter (32 elements) for a lane
constexpr int kMaxWidth = 9856;                      // of an embedding: up to here LDS surely holds the digits of four queries (158 KB)
constexpr int kTileRows = 32;                        // rows of a matrix instruction's other operand

struct Q4Args {
    const uint8_t* packed;      // [N][d / 2]
    const uint16_t* scales;     // [N][d / group], bfloat16
    const float* queries;       // [B][d]
    float* scores;              // [B][ld]
    long long N, ld;
    long long rows, tiles;      // rows of PACK items; tiles of 32 rows
    int B, d, steps;            // steps of a row = elements / 128, rounded up
    int held;                   // tiles whose scores a wave holds back, or 0
};

// A query element as a whole number of 31 bits, in four signed bytes: v = d0 + 2^8 d1 + 2^16 d2 + 2^24 d3.
__device__ __forceinline__ uint32_t four_digits(float x, int shift) {
    const int v = __float2int_rn(ldexpf(x, shift));
    // adding 128 to each byte in turn carries what a byte beyond 127 owes the next one
    return ((uint32_t)v + 0x00808080u) ^ 0x00808080u;
}

// Queries that a pass over the weights serves: up to 8 by BLOCKS pairs, more by SETS eights.
template <int BLOCKS, int SETS> constexpr int queries_of() { return SETS == 1 ? 2 * BLOCKS : 8 * SETS; }

// Scores on the integer matrix cores: both operands are whole numbers and a digit's sums are exact (below 2^21).  Rounded are
// the query (to 2^-31 of a power of two above its largest element: less than float32 there), a group's sum, joined from its
// four digits in float32, and the float32 sum over groups.
// The instruction's 32 rows are eight queries' four digits, its 32 columns rows of weights, its 32 k a quarter of a step, which
// is the smallest group: a lane gets all digits of its sums, and finishes a score with its column's scales.
// Bound by the stream of nibbles, which comes in 16 bytes a lane, 64 neighbouring bytes of sixteen rows an instruction (with
// 8 bytes a lane the same stream reached 4.4 TB/s instead of 5.9).  A lane so has a quarter of row lane % 16 or 16 + lane % 16;
// eight swaps between lanes make of these, for each quarter, column lane % 32 with sixteen k by lane / 32.
// 1.28M items of 512, one query: 70 us with groups of 64, 5.0 TB/s; sixteen, groups of 128: 100 us, 4.2 TB/s with the scores.
// One query's scores are held back in LDS and leave a wave's tiles at a time: stores between the loads cost a long stream more
// than their bytes (5M items of 256: 136 us held back, 143 as they come).  More queries' leave at once (four 159 and 153, eight
// 175 and 164).
// GROUP: weights that share a scale.  PACK: items of a row of weights, 2 for d = 64, whose own rows are half a step: a group's
// sum then belongs to one of the two.  WHOLE: rows are whole steps and their scales aligned.
template <int BLOCKS, int SETS, int GROUP, int PACK, bool WHOLE>
__global__ __launch_bounds__(kThreads, SETS * PACK <= 2 ? 4 : 2) void default_scores_q4_kernel(Q4Args a) {
    constexpr int PARTS = kStep / GROUP, kOf = kQuarters / PARTS;              // groups a step, quarters a group
    constexpr int kQueries = queries_of<BLOCKS, SETS>(), kRows = SETS == 1 ? 8 * BLOCKS : 32;      // digit rows kept of a set
    constexpr int kAhead = 4;                                  // steps whose weights are on their way
    constexpr bool kHold = kQueries == 2 && PACK == 1;
    constexpr int kItems = kTileRows * PACK;                   // of a tile
    static_assert(PACK == 1 || PARTS % PACK == 0, "a group belongs to one item");
    extern __shared__ __align__(16) unsigned char smem[];
    i32x4* digits = reinterpret_cast<i32x4*>(smem);            // [step][quarter][set][half][row]: as the matrix instruction takes them
    float* factor = reinterpret_cast<float*>(digits + (size_t)a.steps * kQuarters * SETS * 2 * kRows);         // [query]
    int* shift = reinterpret_cast<int*>(factor + kQueries);
    float* held = reinterpret_cast<float*>(shift + kQueries);                                    // [wave][tile][items]
    const int groups = a.d * PACK / GROUP;                     // of a row
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int q0 = blockIdx.y * kQueries;

    const int col = lane % 16, h = lane / 16;
    const size_t row_bytes = (size_t)a.d * PACK / 2, bytes = (size_t)a.N * a.d / 2;
    const long long last_row = a.rows - 1, waves = (long long)gridDim.x * kWaves;
    // A wave's work is one sequence of steps, those of a tile and then of the next one.  The weights of kAhead steps are
    // always on their way: waves that all waited for a round of loads would leave the memory idle while they compute.
    typedef uint16_t Scales __attribute__((ext_vector_type(PARTS)));
    const long long first_tile = a.tiles <= waves ? blockIdx.x + (long long)wave * gridDim.x : (long long)blockIdx.x * kWaves + wave;
    uint4 ring_w[kAhead][2];
    Scales ring_s[kAhead];
    long long load_tile = first_tile;
    int load_step = 0;
    auto load = [&](int slot) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            // past the row's end the digits are zero, and past the last item nothing is kept: any weights will do
            size_t at = (size_t)min(load_tile * kTileRows + 16 * u + col, last_row) * row_bytes + min(load_step * (kStep / 2) + 16 * h, (int)row_bytes - 16);
            if (PACK > 1) at = min(at, bytes - 16);
            ring_w[slot][u] = *reinterpret_cast<const uint4*>(a.packed + at);
        }
        // every second step brings the scales of two, a step for each of the column's lanes
        if (load_step % 2 == 0) {
            const size_t first = (size_t)min(load_tile * kTileRows + lane % 32, last_row) * groups;
            const int step = min(load_step + lane / 32, a.steps - 1);
            if constexpr (WHOLE) ring_s[slot] = *reinterpret_cast<const Scales*>(a.scales + first + step * PARTS);
            else {
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    const size_t at = first + min(step * PARTS + p, groups - 1);
                    ring_s[slot][p] = a.scales[PACK > 1 ? min(at, (size_t)a.N * (groups / PACK) - 1) : at];
                }
            }
        }
        if (++load_step == a.steps) { load_step = 0; load_tile += waves; }
    };
    if (first_tile < a.tiles) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(i);              // (while the queries are laid out)
    }

    // factors: a wave per query, or per query in turn
    for (int s = wave; s < kQueries; s += kWaves) {
        uint32_t top = 0;                                      // (magnitudes in the order of their bits)
        if (q0 + s < a.B) {
            const float* phi = a.queries + (size_t)(q0 + s) * a.d;
#pragma unroll 4
            for (int e = lane; e < a.d; e += kWave) top = max(top, __float_as_uint(phi[e]) & 0x7FFFFFFFu);
        }
#pragma unroll
        for (int x = 1; x < kWave; x *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, x));
        const bool odd = top >= 0x7F800000u;                   // an infinity or a NaN
        if (lane == 0) {
            int e = 0;
            if (top > 0 && !odd) (void)frexpf(__uint_as_float(top), &e);           // top < 2^e
            // digits are of x 2^(30 - e); a nibble stands for 16 (n - 8) below.  A query of tiny numbers goes as far as float32 does.
            shift[s] = odd ? 0 : e > -92 ? 30 - e : 122;
            factor[s] = odd ? __builtin_nanf("") : ldexpf(1.0f, e > -92 ? e - 34 : -126);
        }
    }
    __syncthreads();
    // row r of the instruction is digit r % 4 of query r / 4; a lane's sixteen k are neighbouring elements of the quarter, the even
    // and odd ones of each eight apart, as the nibbles of a word come out.  A thread makes a query's four digits of sixteen elements.
    for (int i = threadIdx.x; i < a.steps * kQuarters * 2 * kQueries; i += kThreads) {
        const int q = i % kQueries, half = i / kQueries % 2, quarter = i / kQueries / 2 % kQuarters, step = i / kQueries / 2 / kQuarters;
        const int set = SETS == 1 ? 0 : q / 8, row = (SETS == 1 ? q : q % 8) * 4, first = step * kStep + 32 * quarter + 16 * half;
        uint32_t w[4][4] = {};
        if (q0 + q < a.B && first < a.d * PACK && factor[q] == factor[q]) {     // (d is a multiple of 32: sixteen elements are there or not)
            const float* phi = a.queries + (size_t)(q0 + q) * a.d + (PACK > 1 ? first % a.d : first);
            uint32_t v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = four_digits(phi[e], shift[q]);
#pragma unroll
            for (int e = 0; e < 16; ++e)
#pragma unroll
                for (int digit = 0; digit < 4; ++digit) w[digit][e / 8 * 2 + e % 2] |= ((v[e] >> (8 * digit)) & 255u) << (8 * (e % 8 / 2));
        }
#pragma unroll
        for (int digit = 0; digit < 4; ++digit)
            digits[(((size_t)step * kQuarters + quarter) * SETS + set) * 2 * kRows + half * kRows + row + digit] = i32x4{(int)w[digit][0], (int)w[digit][1], (int)w[digit][2], (int)w[digit][3]};
    }
    __syncthreads();

    float sum[PACK][SETS][BLOCKS];
    auto clear = [&] {
#pragma unroll
        for (int o = 0; o < PACK; ++o)
#pragma unroll
            for (int s = 0; s < SETS; ++s)
#pragma unroll
                for (int k = 0; k < BLOCKS; ++k) sum[o][s][k] = 0.0f;
    };
    clear();
    long long tile = first_tile;
    int step = 0, tiles = 0;
    Scales two_steps = {};
    const int queries = min(kQueries, a.B - q0);
    held += (size_t)wave * a.held * kItems;
    auto release = [&](long long last_tile) {                  // one query's held scores, the last of them of last_tile
        wave_reads_after_writes();
        for (int t = lane / kItems; t < tiles; t += kWave / kItems) {
            const long long item = (last_tile - (long long)(tiles - 1 - t) * waves) * kItems + lane % kItems;
            if (item < a.N) a.scores[(size_t)q0 * a.ld + item] = held[t * kItems + lane % kItems];
        }
        wave_reads_after_writes();
        tiles = 0;
    };
    // (whole rounds of the ring: steps past the wave's last tile are of rows past the last one and leave nothing)
    const int rounds = first_tile < a.tiles ? (int)(((a.tiles - 1 - first_tile) / waves + 1) * a.steps + kAhead - 1) / kAhead : 0;
    for (int round = 0; round < rounds; ++round) {
#pragma unroll
        for (int slot = 0; slot < kAhead; ++slot) {
            __builtin_amdgcn_sched_barrier(0);                 // (steps one after the other: their accumulators share registers)
            uint32_t m[kQuarters][2];                          // column lane % 32, sixteen elements of each quarter
            {
                // rows of sixteen lanes: x[j] has quarters 0 .. 3 of rows 0 .. 15 (A), y[j] those of rows 16 .. 31 (B)
                uint32_t x[4] = {ring_w[slot][0].x, ring_w[slot][0].y, ring_w[slot][0].z, ring_w[slot][0].w};
                uint32_t y[4] = {ring_w[slot][1].x, ring_w[slot][1].y, ring_w[slot][1].z, ring_w[slot][1].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {                  // x: A0 B0 A2 B2, y: A1 B1 A3 B3
                    const auto r = __builtin_amdgcn_permlane16_swap(x[j], y[j], false, false);
                    x[j] = r[0];
                    y[j] = r[1];
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {                  // first and second eight bytes of a quarter: A0 B0 | A0 B0, A2 B2 | A2 B2
                    const auto r = __builtin_amdgcn_permlane32_swap(x[j], x[j + 2], false, false), t = __builtin_amdgcn_permlane32_swap(y[j], y[j + 2], false, false);
                    m[0][j] = r[0]; m[2][j] = r[1];
                    m[1][j] = t[0]; m[3][j] = t[1];
                }
            }
            if (step % 2 == 0) two_steps = ring_s[slot];
            float scale[PARTS];
            uint32_t words[(PARTS + 1) / 2] = {};
            __builtin_memcpy(words, &two_steps, sizeof(Scales));
#pragma unroll
            for (int p = 0; p < PARTS; p += 2) {
                const uint32_t word = (uint32_t)__shfl((int)words[p / 2], lane % 32 + 32 * (step % 2));
                scale[p] = __uint_as_float(word << 16);
                if (p + 1 < PARTS) scale[p + 1] = __uint_as_float(word & 0xFFFF0000u);
            }
            load(slot);
            // a nibble's two's complement of n - 8 in the high half of a byte: 16 (n - 8)
            i32x4 n[kQuarters];
#pragma unroll
            for (int g = 0; g < kQuarters; ++g) {
                const uint32_t v[2] = {m[g][0] ^ 0x88888888u, m[g][1] ^ 0x88888888u};
                n[g] = i32x4{(int)(v[0] << 4 & 0xF0F0F0F0u), (int)(v[0] & 0xF0F0F0F0u), (int)(v[1] << 4 & 0xF0F0F0F0u), (int)(v[1] & 0xF0F0F0F0u)};
            }
            if (tile < a.tiles) {                              // (else past the wave's last tile: 20,000 items of 128, 32 queries 13 us without
                stay_a_branch();                               //  this, 10 with; long streams of wide rows lose 0.7 %)
#pragma unroll
                for (int s = 0; s < SETS; ++s) {
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) {
                        i32x16 acc = {};
#pragma unroll
                        for (int g = p * kOf; g < (p + 1) * kOf; ++g) {
                            // (rows that are not kept repeat others: their sums are not used)
                            const i32x4 x = digits[(((size_t)step * kQuarters + g) * SETS + s) * 2 * kRows + lane / 32 * kRows + lane % kRows];
                            acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, n[g], acc, 0, 0, 0);
                        }
#pragma unroll
                        for (int k = 0; k < BLOCKS; ++k) {
                            const float high = (float)((acc[4 * k + 3] << 8) + acc[4 * k + 2]), low = (float)((acc[4 * k + 1] << 8) + acc[4 * k]);
                            float& to = sum[PACK > 1 ? p / (PARTS / PACK > 0 ? PARTS / PACK : 1) : 0][s][k];
                            to = fmaf(fmaf(high, 65536.0f, low), scale[p], to);
                        }
                    }
                }
            }
            if (++step == a.steps) {
#pragma unroll
                for (int s = 0; s < SETS; ++s)
#pragma unroll
                    for (int k = 0; k < BLOCKS; ++k) {
                        const int q = s * 8 + 2 * k + lane / 32;
                        if (q >= queries) continue;
#pragma unroll
                        for (int o = 0; o < PACK; ++o) {
                            const int at = lane % 32 * PACK + o;
                            const float z = sum[o][s][k] * factor[q];
                            const long long item = tile * kItems + at;
                            if (kHold && a.held > 0) held[tiles * kItems + at] = z;
                            else if (item < a.N) a.scores[(size_t)(q0 + q) * a.ld + item] = z;
                        }
                    }
                if (kHold && a.held > 0 && ++tiles == a.held) release(tile);
                clear();
                step = 0;
                tile += waves;
            }
        }
    }
    if (kHold && tiles > 0) release(tile - waves);
}

// Eight elements a lane; the lanes of a group share its largest absolute value.  Bound by memory, 4.5 bytes an element and the
// scales: 1.28M items of 512 in 660 us, 4.5 TB/s.
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
size_t q4_lds(int queries, int elements) { return (size_t)ceil_div(elements, kStep) * kQuarters * 2 * queries * 4 * 16 + (size_t)queries * 8; }
size_t held_bytes() { return (size_t)kWaves * kTileRows * sizeof(float); }         // a tile of every wave

template <int BLOCKS, int SETS, int GROUP, int PACK, bool WHOLE>
hipError_t go_q4(Q4Args a, hipStream_t st) {
    constexpr int kQueries = queries_of<BLOCKS, SETS>();
    const size_t fixed = q4_lds(kQueries, a.d * PACK), tile = kQueries == 2 && a.B == 1 && PACK == 1 ? held_bytes() : 0;
    a.rows = ceil_div(a.N, PACK);
    a.tiles = ceil_div(a.rows, kTileRows);
    a.steps = (int)ceil_div(a.d * PACK, kStep);
    // (32 queries take 154 to 170 registers a lane, where two workgroups have 128; counted as two, 200,000 items of 128 took 23 us instead of 17)
    const int query_groups = (int)ceil_div(a.B, kQueries), per_cu = SETS == 4 || fixed + tile > kMaxLds / 2 ? 1 : 2;
    // neighbouring tiles to a workgroup's waves; where a wave has one at most, to as many compute units as there are (20,000 items of
    // 512, groups of 64: one query 7.2 and 5.6 us, 32 queries 15.5 and 12.3)
    long long blocks = ceil_div(a.tiles, kWaves);
    if (blocks <= kCUs) blocks = a.tiles < kCUs ? a.tiles : kCUs;
    else if (blocks > (long long)per_cu * kCUs) blocks = (long long)per_cu * kCUs;
    const long long each = ceil_div(a.tiles, blocks * kWaves), room = tile ? (long long)((kMaxLds / per_cu - fixed) / tile) : 0;
    a.held = (int)(each < room ? each : room);
    const size_t lds = fixed + a.held * tile;
    hipError_t e = allow_lds(default_scores_q4_kernel<BLOCKS, SETS, GROUP, PACK, WHOLE>, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((default_scores_q4_kernel<BLOCKS, SETS, GROUP, PACK, WHOLE>), dim3((unsigned)blocks, query_groups), dim3(kThreads), lds, st, a);
    return hipGetLastError();
}

template <int GROUP, int PACK, bool WHOLE>
hipError_t go_q4_sets(const Q4Args& a, hipStream_t st) {
    // as many queries a pass over the weights as there are, up to 32 and what LDS holds of their digits (four always: kMaxWidth)
    int queries = a.B <= 2 ? 2 : a.B <= 4 ? 4 : a.B <= 8 ? 8 : a.B <= 16 ? 16 : 32;
    while (queries > 4 && q4_lds(queries, a.d * PACK) + held_bytes() > kMaxLds) queries /= 2;
    switch (queries) {
        case 2: return go_q4<1, 1, GROUP, PACK, WHOLE>(a, st);
        case 4: return go_q4<2, 1, GROUP, PACK, WHOLE>(a, st);
        case 8: return go_q4<4, 1, GROUP, PACK, WHOLE>(a, st);
        case 16: return go_q4<4, 2, GROUP, PACK, WHOLE>(a, st);
        default: return go_q4<4, 4, GROUP, PACK, WHOLE>(a, st);
    }
}

template <int GROUP>
hipError_t go_q4_group(const Q4Args& a, hipStream_t st) {
    if constexpr (GROUP <= 64) {
        if (a.d == kStep / 2) return go_q4_sets<GROUP, 2, false>(a, st);
    }
    if (GROUP == kStep || (a.d % kStep == 0 && ((uintptr_t)a.scales & 7) == 0)) return go_q4_sets<GROUP, 1, true>(a, st);
    return go_q4_sets<GROUP, 1, GROUP == kStep>(a, st);
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
    if (d > kMaxWidth) return PQ_ERR_UNSUPPORTED;
    if (((uintptr_t)packed & 15) || ((uintptr_t)scales & 1) || (((uintptr_t)queries | (uintptr_t)scores) & 3)) return PQ_ERR_ALIGN;
    const Q4Args a{packed, scales, queries, scores, N, ld, 0, 0, B, d, 0, 0};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return pqk::record_hip_error(group == 32 ? go_q4_group<32>(a, st) : group == 64 ? go_q4_group<64>(a, st) : go_q4_group<128>(a, st));
}

}  // extern "C"
