// A tile of a matrix product C[r][c] = sum_k A(r, k) B(c, k) on the matrix cores, for 16-bit and float32 operands, each of
// them stored either with k running along its rows ("along": element (r, k) at base + r ld + k) or across them ("across":
// element (r, k) at base + k ld + r).
//
// Both operands come to LDS by asynchronous 16-byte loads, three stages of 64 bytes of k (32 16-bit elements, 16 floats), so
// two stages are in flight while one is multiplied.  A stage's chunks of 16 bytes are swapped within their row so that the
// reads of a matrix operand meet every bank: the load picks its source accordingly, as it writes LDS in lane order.
//   along:  [row][4 chunks], chunk c of row r lies at c ^ (r / 4 % 4); an operand is one 16-byte read
//   across: [k][chunks of the rows], 16-bit: chunk c of row k lies at c ^ 4 (k % 4), in rows of eight chunks at c ^ 4 (k / 2 % 2);
//           an operand is two transposing reads
// A lane's operand of a 32x32x16 instruction is eight k of row lane % 32; float32 operands are multiplied in 16-bit pieces.
#pragma once
#include <type_traits>
#include "head_common.hpp"

namespace pqk {
namespace head {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A stage's loads see 2 GB from its first byte on (a tile's rows are at most 256 times 64 KB apart); an offset behind them reads 0.
constexpr uint32_t kBufferBytes = 0x7FFFFFFFu, kPastEnd = 0x80000000u;

constexpr int kStageBytes = 64, kStages = 3;

struct Operand {
    const void* base;
    size_t ld;             // bytes from one stored row to the next
    long long row0;        // first row (r) of the tile
    long long rows;        // rows there are: past the last one the last is read again
    long long k0, k1;      // range of k: past k1 zeros are read
    int block = 0;         // along: a stored row holds this many k (a multiple of a stage's, as k0 is), the next ones lie
    size_t to_next = 0;    //   to_next bytes on; 0: all of them
    int again = 0;         // along, row0 = 0: rows from this one on are the first ones again; 0: none
};

// acc[mi][ni] += x[mi] y[ni], 16-bit operands of sixteen k.
template <typename T, int MI, int NI>
__device__ __forceinline__ void multiply(const s16x8 (&x)[MI], const s16x8 (&y)[NI], f32x16 (&acc)[MI][NI]) {
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) {
            if constexpr (std::is_same<T, _Float16>::value)
                acc[mi][ni] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x[mi]), __builtin_bit_cast(f16x8, y[ni]), acc[mi][ni], 0, 0, 0);
            else
                acc[mi][ni] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x[mi]), __builtin_bit_cast(bf16x8, y[ni]), acc[mi][ni], 0, 0, 0);
        }
}

// Eight floats as the sums of three bfloat16 each, x = p0 + p1 + p2 (each piece is what the ones before it leave, rounded to nearest:
// 24 bits are 8 and 8 and 8).  For x of 1 to 2 a piece leaves at most 2^-8, then 2^-17, then nothing.
struct Pieces { s16x8 p[3]; };
__device__ __forceinline__ Pieces pieces_of(s16x8 a, s16x8 b) {
    const f32x4 u = __builtin_bit_cast(f32x4, a), v = __builtin_bit_cast(f32x4, b);
    float x[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
    Pieces r;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), bf16x2));
            if (k < 2) {
                x[2 * i] -= __builtin_bit_cast(float, w[i] << 16);
                x[2 * i + 1] -= __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
            }
        }
        r.p[k] = __builtin_bit_cast(s16x8, w);
    }
    return r;
}

// The same for sixteen k of float32, x and y holding four k each.  A product is six of its pieces', all but the smallest
// (p1 q2, p2 q1, p2 q2: together below 2^-24 |x y|, as p1 is at most 2^-8 and p2 2^-17 of a power of two below x), the small ones first.  Six
// instructions of the 16-bit rate take 37 % of the time of the eight float32 ones: 208 against 146 TFLOP/s at 4096^3.
template <int MI, int NI>
__device__ __forceinline__ void multiply_floats(const s16x8 (&x)[2][MI], const s16x8 (&y)[2][NI], f32x16 (&acc)[MI][NI]) {
    constexpr int order[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
    Pieces q[NI];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) q[ni] = pieces_of(y[0][ni], y[1][ni]);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
        const Pieces p = pieces_of(x[0][mi], x[1][mi]);
#pragma unroll
        for (int o = 0; o < 6; ++o)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
                acc[mi][ni] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, p.p[order[o][0]]), __builtin_bit_cast(bf16x8, q[ni].p[order[o][1]]),
                                                                      acc[mi][ni], 0, 0, 0);
    }
}

// ROWS rows of an operand, as a workgroup of THREADS brings them to LDS and its waves read them.
template <typename T, int ROWS, bool ALONG, int THREADS>
struct Side {
    static constexpr int kBytes = ROWS * kStageBytes;                      // of a stage
    static constexpr int kK = kStageBytes / (int)sizeof(T);                // k of a stage
    static constexpr int kRowChunks = ROWS * (int)sizeof(T) / 16;          // across: chunks of a stored row
    static constexpr int kLoads = kBytes / 16 / THREADS;                   // asynchronous loads of a thread and stage
    static_assert(ROWS >= 64, "rows of at least eight chunks");
    static_assert(kBytes % (16 * THREADS) == 0, "every wave loads as much");

    const char* base;                                                      // moves on stage by stage
    size_t ld;
    uint32_t offset[kLoads];
    long long k, k1;
    int block;
    size_t to_next;

    int tid;

    __device__ __forceinline__ void start(const Operand& o) {
        tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                                      // (so that a loop over tiles does not keep all this in registers meanwhile)
        k = o.k0; k1 = o.k1; ld = o.ld; block = o.block; to_next = o.to_next;
        if constexpr (ALONG) base = static_cast<const char*>(o.base) + (size_t)o.row0 * ld + (block ? (size_t)(o.k0 / block) * to_next + (size_t)(o.k0 % block) * sizeof(T) : (size_t)o.k0 * sizeof(T));
        else base = static_cast<const char*>(o.base) + (size_t)o.k0 * ld + (size_t)o.row0 * sizeof(T);
        const int last = (int)min((long long)ROWS, o.rows - o.row0) - 1;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at = (tid / kWave * kLoads + i) * kWave + tid % kWave;
            if constexpr (ALONG) {
                const int row = at / 4, chunk = (at % 4) ^ (row / 4 % 4);
                offset[i] = (uint32_t)min(o.again && row >= o.again ? row - o.again : row, last) * (uint32_t)ld + (uint32_t)chunk * 16u;
            } else {
                const int kk = at / kRowChunks, chunk = swap(at % kRowChunks, kk), most = last * (int)sizeof(T) / 16;
                offset[i] = (uint32_t)kk * (uint32_t)ld + (uint32_t)min(chunk, most) * 16u;
            }
        }
    }
    static __device__ __forceinline__ int swap(int chunk, int kk) {
        return sizeof(T) != 2 ? chunk : kRowChunks >= 16 ? chunk ^ (4 * (kk % 4)) : chunk ^ (4 * (kk / 2 % 2));
    }

    // How many stages from k0 on hold nothing but operand.
    static __device__ __forceinline__ int whole_stages(const Operand& o) { return (int)((o.k1 - o.k0) / kK); }

    // The next stage, on its way; CHECKED: it may end, or lie, behind k1 (zeros).
    template <bool CHECKED>
    __device__ __forceinline__ void load(unsigned char* stage) {
        unsigned char* to = stage + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * (kLoads * kWave * 16);
        // (as a buffer, whose offsets past the end read zeros; the compiler then also counts these loads one by one, where it
        // waits for all of them to be done if they are global loads)
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, kBufferBytes, 0x00020000);
        auto bring = [&](int i, uint32_t at) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to + i * kWave * 16), 16, at, 0, 0, 0);
        };
        if (!CHECKED || k + kK <= k1) {                                    // (the same for all lanes)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) bring(i, offset[i]);
        } else {
            stay_a_branch();
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int at = (tid / kWave * kLoads + i) * kWave + tid % kWave;
                const int kk = ALONG ? ((at % 4) ^ (at / 4 / 4 % 4)) * (16 / (int)sizeof(T)) : at / kRowChunks;
                bring(i, k + kk >= k1 ? kPastEnd : offset[i]);
            }
        }
        k += kK;
        base += ALONG ? (size_t)kStageBytes : (size_t)kK * ld;
        if (ALONG && block && k % block == 0) base += to_next - (size_t)block * sizeof(T);
    }

    // rows row0 .. + 31: 16-bit, the operand of the u-th half of the stage; float32, the u-th half of the lane's eight k
    static __device__ __forceinline__ s16x8 read(const unsigned char* stage, int row0, int u) {
        const int lane = threadIdx.x % kWave;
        if constexpr (ALONG) {
            const int row = row0 + lane % 32;
            const int chunk = sizeof(T) == 2 ? 2 * u + lane / 32 : 2 * (lane / 32) + u;
            return *reinterpret_cast<const s16x8*>(stage + row * kStageBytes + ((chunk ^ (row / 4 % 4)) * 16));
        } else if constexpr (sizeof(T) == 2) {
            // sixteen lanes read four stored rows of sixteen elements and get a column each
            const int kk = 16 * u + 8 * (lane / 32) + lane % 16 / 4, row = row0 + 16 * (lane / 16 % 2) + 4 * (lane % 4);
            const unsigned char* p = stage + kk * (ROWS * 2) + (swap(row / 8, kk) * 16) + row % 8 * 2;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 4 * (ROWS * 2)));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            const unsigned char* p = stage + (8 * (lane / 32) + 4 * u) * (ROWS * 4) + (row0 + lane % 32) * 4;
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const float*>(p + i * (ROWS * 4));
            return __builtin_bit_cast(s16x8, v);
        }
    }
};

// An array per stage and side: the compiler tells loads into one from reads of another, and waits for no more than it must.
// (Tiles of equal sizes in one kernel share them.)
template <int WHICH, int BYTES>
__device__ __forceinline__ unsigned char* stage_memory() {
    __shared__ __align__(16) unsigned char memory[BYTES];
    return memory;
}

// BM x BN tile by waves in a grid of (BM / WM) x (BN / WN).  acc[mi][ni][i] is row 32 mi + 8 (i / 4) + 4 (lane / 32) + i % 4,
// column 32 ni + lane % 32 of the wave's part.
template <typename T, int BM, int BN, int WM, int WN, bool A_ALONG, bool B_ALONG>
struct MatrixTile {
    static constexpr int kThreads = BM / WM * (BN / WN) * kWave;
    static constexpr int MI = WM / 32, NI = WN / 32;
    using A = Side<T, BM, A_ALONG, kThreads>;
    using B = Side<T, BN, B_ALONG, kThreads>;

    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); }
    static __device__ __forceinline__ int wave_row() { return wave() / (BN / WN) * WM; }
    static __device__ __forceinline__ int wave_col() { return wave() % (BN / WN) * WN; }

    // Between products: 4 KB of LDS for a wave alone, to lay blocks of its part out in rows (tiles with a side of 256, and 64 x 64).
    static __device__ __forceinline__ unsigned char* own_memory() {
        if constexpr (BM == 64 && BN == 64) {
            static_assert(kThreads == 4 * kWave, "a stage for each of four waves");
            return wave() < 2 ? (wave() == 0 ? stage_memory<0, A::kBytes>() : stage_memory<1, A::kBytes>())
                              : (wave() == 2 ? stage_memory<3, B::kBytes>() : stage_memory<4, B::kBytes>());
        } else if constexpr (BM == 256) {
            return (wave() < 4 ? stage_memory<0, A::kBytes>() : stage_memory<1, A::kBytes>()) + wave() % 4 * 4096;
        } else {
            static_assert(BN == 256, "a stage for four waves");
            return (wave() < 4 ? stage_memory<3, B::kBytes>() : stage_memory<4, B::kBytes>()) + wave() % 4 * 4096;
        }
    }

    static __device__ __forceinline__ void run(const Operand& oa, const Operand& ob, f32x16 (&acc)[MI][NI]) {
        unsigned char *a0 = stage_memory<0, A::kBytes>(), *a1 = stage_memory<1, A::kBytes>(), *a2 = stage_memory<2, A::kBytes>();
        unsigned char *b0 = stage_memory<3, B::kBytes>(), *b1 = stage_memory<4, B::kBytes>(), *b2 = stage_memory<5, B::kBytes>();
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x16{};
        A a;
        B b;
        a.start(oa);
        b.start(ob);
        const int steps = (int)((oa.k1 - oa.k0 + A::kK - 1) / A::kK);
        const int row0 = wave_row(), col0 = wave_col();

        auto load = [&](int stage, auto checked) {
            a.template load<decltype(checked)::value>(stage == 0 ? a0 : stage == 1 ? a1 : a2);
            b.template load<decltype(checked)::value>(stage == 0 ? b0 : stage == 1 ? b1 : b2);
        };
        auto step = [&](auto stage_c, auto checked) {
            constexpr int stage = decltype(stage_c)::value;
            const unsigned char* sa = stage == 0 ? a0 : stage == 1 ? a1 : a2;
            const unsigned char* sb = stage == 0 ? b0 : stage == 1 ? b1 : b2;
            // this stage's loads are done when only the next one's are in flight; past the barrier that holds for every
            // wave, and every wave is done with the stage that is loaded next
            wait_loads<A::kLoads + B::kLoads>();
            s16x8 x[2][MI], y[2][NI];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) x[u][mi] = A::read(sa, row0 + 32 * mi, u);
#pragma unroll
                for (int ni = 0; ni < NI; ++ni) y[u][ni] = B::read(sb, col0 + 32 * ni, u);
            }
            __builtin_amdgcn_sched_barrier(0);                 // (reads behind a load into LDS would wait for that load)
            load((stage + 2) % 3, checked);
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int u = 0; u < 2; ++u) multiply<T, MI, NI>(x[u], y[u], acc);
            } else multiply_floats<MI, NI>(x, y, acc);
        };
        using std::integral_constant;
        // Two stages more than there are get loaded (zeros): the count of loads in flight is the same in every step, and the
        // compiler, which counts them too, finds nothing else to wait for.  The loads of a step whose stages are whole are
        // free of branches, and go out between its matrix instructions.
        load(0, std::true_type{});
        load(1, std::true_type{});
        const int whole = min(A::whole_stages(oa), B::whole_stages(ob));
        int s = 0;
        for (; s + 4 < whole; s += 3) {
            step(integral_constant<int, 0>{}, std::false_type{});
            step(integral_constant<int, 1>{}, std::false_type{});
            step(integral_constant<int, 2>{}, std::false_type{});
        }
        while (s < steps) {
            step(integral_constant<int, 0>{}, std::true_type{});
            if (++s >= steps) break;
            step(integral_constant<int, 1>{}, std::true_type{});
            if (++s >= steps) break;
            step(integral_constant<int, 2>{}, std::true_type{});
            ++s;
        }
        wait_loads<0>();                                       // nothing is on its way to LDS, or being read there, any more
    }

    // All but the wave's last LEFT loads have arrived and its LDS reads are done; then the workgroup's barrier.
    template <int LEFT>
    static __device__ __forceinline__ void wait_loads() {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
    }
};

}  // namespace head
}  // namespace pqk
