// pq_default_log_probs: checks, pieces and the entry point (the kernels: default_log_probs.hpp).
#include "default_log_probs.hpp"

namespace pqk {
namespace head {
namespace {

// How many candidates for the K best are scored in 64 bits at least: float32 scores may put neighbours in another order, not items that far apart
// (neighbours among the best 100 of 1.28M lie some 1e-3 of their scores apart, a sum's rounding 1e-6).
int keep_of(int K) { return K ? K + 16 + K / 8 : 0; }
static_assert(PQ_MAX_K + 16 + PQ_MAX_K / 8 + (PQ_MAX_K + 16 + PQ_MAX_K / 8) / 4 + 32 <= kMostKept, "a cut leaves no more");

struct Layout {
    Passes pieces;
    int groups;
    size_t keys_at, count_at, floor_at, bytes;
};
Layout lay_out(long long N, int B, int d, int type, int K) {
    Layout l;
    l.pieces = pieces_of(N, B, keep_of(K));
    l.groups = 0;
    for (long long done = 0; done < N; done += l.pieces.after(done)) l.groups += plan_dense(l.pieces.after(done), B, d, type).groups;
    l.keys_at = round_up((size_t)l.groups * B * sizeof(float4), 256);
    l.count_at = l.keys_at + l.pieces.key_bytes(B);
    l.floor_at = l.count_at + (K ? round_up((size_t)B * sizeof(int), 256) : 0);
    l.bytes = l.floor_at + (K ? round_up((size_t)B * sizeof(float), 256) : 0);
    return l;
}

int check(long long N, int B, int d, int type, int K) {
    if (K < 0 || K > N) return PQ_ERR_SHAPE;
    const int rc = check_dense(N, B, d, type);
    return rc != PQ_OK ? rc : K > PQ_MAX_K ? PQ_ERR_UNSUPPORTED : PQ_OK;
}

template <typename T>
hipError_t pass(const Layout& l, DenseProbsArgs a, DenseFinishArgs f, int type, hipStream_t st) {
    hipError_t e = hipSuccess;
    for (long long done = 0; done < a.N && e == hipSuccess; done = a.end) {
        const DensePlan p = plan_dense(l.pieces.after(done), a.B, a.d, type);
        a.first = done;
        a.end = done + l.pieces.after(done);
        a.store = f.K != 0 && done == 0;
        a.item_tiles = p.item_tiles; a.tiles_each = p.tiles_each; a.groups = p.groups; a.position_tiles = p.position_tiles;
        e = dense_probs<T>(p, a, st);
        a.partial += (size_t)p.groups * a.B;
        if (e == hipSuccess && f.K && a.end < a.N) e = launch_select(a.lists, a.B, done == 0 ? (int)a.end : 0, st);
    }
    return e != hipSuccess ? e : dense_probs_finish<T>(f, st);
}

}  // namespace
}  // namespace head
}  // namespace pqk

using namespace pqk::head;

extern "C" {

size_t pq_default_log_probs_workspace_bytes(long long N, int B, int d, int type, int K) {
    return check(N, B, d, type, K) == PQ_OK ? lay_out(N, B, d, type, K).bytes : 0;
}

int pq_default_log_probs(const void* W, const void* queries, const int* items, long long N, int B, int d, int type, int n, int K, float temperature,
                         float* log_probs, float* entropy, float* lse, int* top_items, float* top_log_probs, void* workspace, size_t workspace_bytes,
                         void* stream) {
    if (!W || !queries || !entropy || !lse || !workspace || (n != 0 && (!items || !log_probs)) || (K != 0 && (!top_items || !top_log_probs))) return PQ_ERR_NULL;
    if (n < 0 || !(temperature > 0.0f)) return PQ_ERR_SHAPE;
    const int rc = check(N, B, d, type, K);
    if (rc != PQ_OK) return rc;
    if (n > kMostGiven || !temperature_fits(temperature)) return PQ_ERR_UNSUPPORTED;
    if ((((uintptr_t)W | (uintptr_t)queries | (uintptr_t)workspace) & 15) || (((uintptr_t)entropy | (uintptr_t)lse) & 3) ||
        (n && (((uintptr_t)items | (uintptr_t)log_probs) & 3)) || (K && (((uintptr_t)top_items | (uintptr_t)top_log_probs) & 3)))
        return PQ_ERR_ALIGN;
    const Layout l = lay_out(N, B, d, type, K);
    if (workspace_bytes < l.bytes) return PQ_ERR_WORKSPACE;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    DenseProbsArgs a{};
    a.W = W; a.H = queries; a.N = N; a.B = B; a.d = d; a.scale = (float)(kLog2eDouble / temperature);
    a.partial = reinterpret_cast<float4*>(ws);
    a.lists = Lists{reinterpret_cast<uint64_t*>(ws + l.keys_at), reinterpret_cast<int*>(ws + l.count_at), reinterpret_cast<float*>(ws + l.floor_at),
                    (uint32_t)l.pieces.cap, l.pieces.keep};
    const DenseFinishArgs f{W, queries, items, N, B, d, n, K, temperature, a.partial, l.groups, l.pieces.first == N ? (int)N : 0, a.lists,
                            log_probs, entropy, lse, top_items, top_log_probs};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return pqk::record_hip_error(type == PQ_FLOAT32 ? pass<float>(l, a, f, type, st) : type == PQ_BFLOAT16 ? pass<__bf16>(l, a, f, type, st) : pass<_Float16>(l, a, f, type, st));
}

}  // extern "C"
