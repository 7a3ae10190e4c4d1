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
constexpr int kStep = 64;                            // elements of an embedding per matrix instruction
constexpr int kTileItems = 16;

struct Q4Args {
    const uint8_t* packed;      // [N][d / 2]
    const uint16_t* scales;     // [N][d / group], bfloat16
    const float* queries;       // [B][d]
    float* scores;              // [B][ld]
    long long N, ld, item_tiles;
    int B, d, steps;            // steps = d / 64, rounded up
};

// What LDS holds, for SETS sets of four queries: the queries' digits as the matrix instruction takes them, what the
// nibbles' offset of 8 adds to each group, and a factor per query.
struct Q4Lds {
    i32x4* digits;              // [step][part][set][lane]
    i32x4* offsets;             // [group][set][query of the set]
    float* factor;              // [set * 4 + query]
};

// A query element as a whole number of 31 bits, in four signed bytes: v = d0 + 2^8 d1 + 2^16 d2 + 2^24 d3.
__device__ __forceinline__ uint32_t four_digits(float x, int shift) {
    const int v = __float2int_rn(ldexpf(x, shift));
    // adding 128 to each byte in turn carries what a byte beyond 127 owes the next one
    return ((uint32_t)v + 0x00808080u) ^ 0x00808080u;
}

// Scores on the integer matrix cores: both operands are exact, so are the sums of a group (below 2^24), and what is rounded
// is the query (to 2^-31 of its largest element, less than its float32 rounding there) and the float32 sum over groups.
// The instruction's 16 rows are four queries' four digits, its 16 columns items: a lane finishes one score, all its digits
// at hand, with its item's scale.
// Bound by the stream of nibbles: per 16 weights a lane spends six instructions on unpacking, one matrix instruction for
// four queries and eight more a group, which the memory hides up to some 32 queries.  PARTS = 2 (groups of 32): two groups
// share a step; each gets the step's digits with the other's zeroed.
template <int SETS, int GROUP, int TILES>
__global__ __launch_bounds__(kThreads) void default_scores_q4_kernel(Q4Args a) {
    constexpr int PARTS = GROUP == 32 ? 2 : 1, PER_GROUP = GROUP > kStep ? GROUP / kStep : 1;   // groups a step, steps a group
    constexpr int kAhead = 8;                                  // steps whose weights a lane has asked for
    extern __shared__ __align__(16) unsigned char smem[];
    const int groups = a.d / GROUP;
    Q4Lds L;
    L.digits = reinterpret_cast<i32x4*>(smem);
    L.offsets = L.digits + (size_t)a.steps * PARTS * SETS * kWave;
    L.factor = reinterpret_cast<float*>(L.offsets + (size_t)groups * SETS * 4);
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int q0 = blockIdx.y * SETS * 4;

    // factors: one wave per query in turn
    int* shift = reinterpret_cast<int*>(L.factor + SETS * 4);
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
            shift[s] = any_odd ? 0 : 30 - e;
            L.factor[s] = any_odd ? __builtin_nanf("") : ldexpf(1.0f, e > -96 ? e - 30 : -126);
            if (e <= -96) shift[s] = 126;                                // (a query of tiny numbers: as far as float32 goes)
        }
    }
    __syncthreads();
    // digits: row r of the instruction is digit r % 4 of query r / 4; a lane's 16 bytes are elements 16 (lane / 16) .. + 15
    // of the step, the even and odd ones of each eight apart, as the nibbles of a word come out
    for (int i = threadIdx.x; i < a.steps * SETS * kWave; i += kThreads) {
        const int l = i % kWave, set = i / kWave % SETS, step = i / kWave / SETS;
        const int row = l % 16, q = set * 4 + row / 4, first = step * kStep + 16 * (l / 16);
        const bool live = q0 + q < a.B && first < a.d;                   // (d is a multiple of 32: sixteen elements are there or not)
        i32x4 v = {0, 0, 0, 0};
        if (live && L.factor[q] == L.factor[q]) {
            const float* phi = a.queries + (size_t)(q0 + q) * a.d + first;
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t byte = (four_digits(phi[e], shift[q]) >> (8 * (row % 4))) & 255u;
                w[e / 8 * 2 + e % 2] |= byte << (8 * (e % 8 / 2));
            }
            v = i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
        }
        const i32x4 none = {0, 0, 0, 0};
        if (PARTS == 1) L.digits[((size_t)step * SETS + set) * kWave + l] = v;
        else {
            L.digits[((size_t)(step * 2) * SETS + set) * kWave + l] = l < 32 ? v : none;
            L.digits[((size_t)(step * 2 + 1) * SETS + set) * kWave + l] = l < 32 ? none : v;
        }
    }
    // what the offset of 8 makes of a group: -8 times its digits' sums
    for (int i = threadIdx.x; i < groups * SETS * 4; i += kThreads) {
        const int q = i % (SETS * 4), g = i / (SETS * 4);
        int sum[4] = {0, 0, 0, 0};
        if (q0 + q < a.B && L.factor[q] == L.factor[q]) {
            const float* phi = a.queries + (size_t)(q0 + q) * a.d + (size_t)g * GROUP;
            for (int e = 0; e < GROUP; ++e) {
                const uint32_t four = four_digits(phi[e], shift[q]);
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r] += (int)(int8_t)(four >> (8 * r));
            }
        }
        L.offsets[i] = i32x4{-8 * sum[0], -8 * sum[1], -8 * sum[2], -8 * sum[3]};
    }
    __syncthreads();

    const int col = lane % 16, h = lane / 16;
    const size_t row_bytes = (size_t)a.d / 2;
    const long long last_item = a.N - 1, waves = (long long)gridDim.x * kWaves;
    for (long long t = (long long)blockIdx.x * kWaves + wave; t * TILES < a.item_tiles; t += waves) {
        const uint8_t* row[TILES];
        const uint16_t* scale[TILES];
#pragma unroll
        for (int u = 0; u < TILES; ++u) {
            const long long item = min((t * TILES + u) * kTileItems + col, last_item);
            row[u] = a.packed + (size_t)item * row_bytes;
            scale[u] = a.scales + (size_t)item * groups;
        }
        float sum[TILES][SETS];
#pragma unroll
        for (int u = 0; u < TILES; ++u)
#pragma unroll
            for (int s = 0; s < SETS; ++s) sum[u][s] = 0.0f;
        for (int step0 = 0; step0 < a.steps; step0 += kAhead) {
            uint2 w[kAhead][TILES];
            uint16_t sc[kAhead / PER_GROUP * PARTS][TILES];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                // past the row's end the digits are zero: any weights will do
                const int at = min((step0 + i) * (kStep / 2) + 8 * h, (int)row_bytes - 8);
#pragma unroll
                for (int u = 0; u < TILES; ++u) w[i][u] = *reinterpret_cast<const uint2*>(row[u] + at);
            }
#pragma unroll
            for (int i = 0; i < kAhead / PER_GROUP * PARTS; ++i) {
                const int g = min(step0 / PER_GROUP * PARTS + i, groups - 1);
#pragma unroll
                for (int u = 0; u < TILES; ++u) sc[i][u] = scale[u][g];
            }
            i32x4 acc[TILES][SETS];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (step0 + i < a.steps) {
                    i32x4 n[TILES];
#pragma unroll
                    for (int u = 0; u < TILES; ++u) {
                        const uint2 v = w[i][u];
                        n[u] = i32x4{(int)(v.x & 0x0F0F0F0Fu), (int)(v.x >> 4 & 0x0F0F0F0Fu), (int)(v.y & 0x0F0F0F0Fu), (int)(v.y >> 4 & 0x0F0F0F0Fu)};
                    }
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) {
                        const int g = (step0 + i) / PER_GROUP * PARTS + p;
                        if (PARTS == 2 && g >= groups) continue;         // (d = 32 mod 64: the last step holds one group)
#pragma unroll
                        for (int s = 0; s < SETS; ++s) {
                            const i32x4 q = L.digits[((size_t)((step0 + i) * PARTS + p) * SETS + s) * kWave + lane];
                            if (i % PER_GROUP == 0) {
                                const i32x4 c = L.offsets[((size_t)g * SETS + s) * 4 + h];
#pragma unroll
                                for (int u = 0; u < TILES; ++u) acc[u][s] = c;
                            }
#pragma unroll
                            for (int u = 0; u < TILES; ++u) acc[u][s] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q, n[u], acc[u][s], 0, 0, 0);
                            if (i % PER_GROUP == PER_GROUP - 1) {
#pragma unroll
                                for (int u = 0; u < TILES; ++u) {
                                    const i32x4 v = acc[u][s];
                                    float x = fmaf((float)v[3], 256.0f, (float)v[2]);
                                    x = fmaf(x, 256.0f, (float)v[1]);
                                    x = fmaf(x, 256.0f, (float)v[0]);
                                    const float by = __uint_as_float((uint32_t)sc[(i / PER_GROUP) * PARTS + p][u] << 16);
                                    sum[u][s] = fmaf(x, by, sum[u][s]);
                                }
                            }
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < TILES; ++u) {
            const long long item = (t * TILES + u) * kTileItems + col;
#pragma unroll
            for (int s = 0; s < SETS; ++s) {
                const int q = s * 4 + h;
                if (item < a.N && q0 + q < a.B) a.scores[(size_t)(q0 + q) * a.ld + item] = sum[u][s] * L.factor[q];
            }
        }
    }
}

// Eight elements a lane; the lanes of a group share its largest absolute value.  A stream of 4 N d bytes in.
__global__ __launch_bounds__(256) void quantise_items_kernel(const float* W, long long pieces, int lanes_per_group, uint32_t* packed, uint16_t* scales) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (long long)gridDim.x * 256) {
        const float4 x = reinterpret_cast<const float4*>(W)[2 * i], y = reinterpret_cast<const float4*>(W)[2 * i + 1];
        const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
        // (a group's lanes are neighbours of one wave and run this together: the pieces are a multiple of a group's)
        for (int s = 1; s < lanes_per_group; s *= 2) top = fmaxf(top, __shfl_xor(top, s));
        // the scale is rounded to bfloat16 (nearest even) first, the weights then to multiples of what is kept
        const uint32_t bits = __float_as_uint(top / 7.0f);
        const uint32_t kept = (bits + 0x7FFFu + (bits >> 16 & 1u)) >> 16;
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

size_t q4_lds(int sets, int d, int group) {
    const size_t steps = (size_t)ceil_div(d, kStep);
    return steps * (group == 32 ? 2 : 1) * sets * kWave * 16 + (size_t)(d / group) * sets * 64 + (size_t)sets * 4 * 8;
}

template <int SETS, int GROUP>
hipError_t go_q4(Q4Args a, hipStream_t st) {
    constexpr int TILES = 2;
    const size_t lds = q4_lds(SETS, a.d, GROUP);
    const long long tiles = ceil_div(a.N, kTileItems);
    a.item_tiles = tiles;
    const int query_groups = (int)ceil_div(a.B, SETS * 4), per_cu = lds > kMaxLds / 2 ? 1 : 2;
    long long blocks = ceil_div(tiles, (long long)TILES * kWaves);
    if (blocks > (long long)per_cu * kCUs) blocks = (long long)per_cu * kCUs;
    hipError_t e = allow_lds(default_scores_q4_kernel<SETS, GROUP, TILES>, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((default_scores_q4_kernel<SETS, GROUP, TILES>), dim3((unsigned)blocks, query_groups), dim3(kThreads), lds, st, a);
    return hipGetLastError();
}

template <int GROUP>
hipError_t go_q4_sets(const Q4Args& a, hipStream_t st) {
    // as many queries a pass over the weights as there are, up to 32 and what LDS holds of their digits
    int sets = a.B <= 4 ? 1 : a.B <= 8 ? 2 : a.B <= 16 ? 4 : 8;
    while (sets > 1 && q4_lds(sets, a.d, GROUP) > kMaxLds) sets /= 2;
    return sets == 8 ? go_q4<8, GROUP>(a, st) : sets == 4 ? go_q4<4, GROUP>(a, st) : sets == 2 ? go_q4<2, GROUP>(a, st) : go_q4<1, GROUP>(a, st);
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
    if (q4_lds(1, d, group) > kMaxLds) return PQ_ERR_UNSUPPORTED;
    if (((uintptr_t)packed & 15) || ((uintptr_t)scales & 1) || (((uintptr_t)queries | (uintptr_t)scores) & 3)) return PQ_ERR_ALIGN;
    const Q4Args a{packed, scales, queries, scores, N, ld, 0, B, d, (int)ceil_div(d, kStep)};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return pqk::record_hip_error(group == 32 ? go_q4_sets<32>(a, st) : group == 64 ? go_q4_sets<64>(a, st) : go_q4_sets<128>(a, st));
}

}  // extern "C"
