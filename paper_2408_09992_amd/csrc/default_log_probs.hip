// pq_default_log_probs: checks, pieces and the entry point (the kernels: default_log_probs.hpp).
#include "default_log_probs.hpp"

namespace pqk {
namespace head {
namespace {

// How many candidates for the K best are scored in 64 bits at least: float32 scores may put neighbours in another order, not items that far apart
// (neighbours among the best 100 of 1.28M lie some 1e-3 of their scores apart, a sum's rounding 1e-6).  A number and no bound: of more than 16 items beyond the K-th within that
// rounding, near copies of one item, it decides which are among the candidates.
int keep_of(int K) { return K ? K + 16 : 0; }
static_assert(most_of(PQ_MAX_K + 16) < kMostKept, "a cut leaves no more");

// The cross entropy's plan of a piece, whose lists have no more regions than there are places for: how many these are, and the places of each.
DensePlan plan_piece(long long items, int B, int d, int type, bool listed, int& regions, long long& region) {
    DensePlan p = plan_dense(items, B, d, type);
    const int shares = shares_of(p);
    if (p.few) region = ceil_div(ceil_div(items, few_items(d)), p.groups) * few_items(d);
    else {
        if (listed && (long long)p.groups * shares > kMostRegions) {
            // the rounds over the chip that take least, a tile of items a unit; of as good ones the fewest groups
            // (two workgroups a compute unit of those that leave room for it: one alone has nothing to do while its candidates are on their way; 1.28M items of 64 bfloat16,
            // 100 positions, K = 10 and 100: 161 and 229 us by one, 121 and 160 by two)
            const int slots = p.positions == 256 ? kCUs : 2 * kCUs;
            double best = 1e300;
            const long long least = ceil_div(p.item_tiles * shares, kMostRegions);
            for (long long each = least; each <= 2 * least + 16; ++each) {
                const double cost = (double)ceil_div(ceil_div(p.item_tiles, each) * p.position_tiles, slots) * (each + 0.1);
                if (cost <= best) { best = cost; p.tiles_each = (int)each; }
            }
            p.groups = (int)ceil_div(p.item_tiles, p.tiles_each);
        }
        if (listed) p.tiles_each = (int)ceil_div(p.item_tiles, p.groups);         // (as many places as the groups have tiles, and few more)
        region = (long long)p.tiles_each * p.loss_items / shares;
    }
    regions = p.groups * shares;
    return p;
}

struct Layout : ListLayout {
    Passes passes;
    Sums sums;
};
Layout lay_out(long long N, int B, int d, int type, int K) {
    Layout l;
    // (few positions' candidates wait in LDS: 64 positions of 1.28M items of 128, K = 100, one piece after the first 187 us, two 145)
    l.passes = passes_of(N, B, keep_of(K), plan_dense(N, B, d, type).few ? 0.8 * kFewWaiting * kCUs : 1e300);
    for (long long done = 0, now, region; done < N; done += now) {
        int regions;
        now = l.passes.after(done);
        l.sums.piece(plan_piece(now, B, d, type, K != 0, regions, region).groups);
        l.piece(done == 0 ? now : regions * region);
    }
    l.sums.lay_out(B);
    l.ListLayout::lay_out(l.sums.bytes(B), B, l.passes);
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
        const long long now = l.passes.after(done);
        const DensePlan p = plan_piece(now, a.B, a.d, type, f.K != 0, f.regions, a.region);
        a.first = done;
        a.end = done + now;
        a.store = f.K != 0 && done == 0;
        a.item_tiles = p.item_tiles; a.tiles_each = p.tiles_each; a.groups = p.groups; a.position_tiles = p.position_tiles;
        e = dense_probs<T>(p, a, st);
        l.sums.advance(p.groups, a.done, a.written);
        if (e == hipSuccess && f.K && a.end < a.N) e = launch_select(a.lists, a.B, a.store ? (int)now : 0, f.regions, a.region, st);
        f.stored = a.store ? (int)now : 0;
        f.region = a.region;
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
    a.partials = l.sums.slots;
    a.lists = l.lists(ws, l.passes.keep);
    const DenseFinishArgs f{W, queries, items, N, B, d, n, K, 1.0 / temperature, 1.0 / base_of(a.scale, temperature), a.partial, l.sums.slots, 0, 0, 0, a.lists, log_probs, entropy, lse, top_items, top_log_probs};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return pqk::record_hip_error(type == PQ_FLOAT32 ? pass<float>(l, a, f, type, st) : type == PQ_BFLOAT16 ? pass<__bf16>(l, a, f, type, st) : pass<_Float16>(l, a, f, type, st));
}

}  // extern "C"
