"""Log-probabilities, entropy and the likeliest items of the whole catalogue, by sub-ids and by W phi, against the definitions in 64 bits.

u = 2^-24 is float32's unit.  A float32 score is off by at most (m - 1) u (by sub-ids) or (d + 2) u (W phi) times the sum of its terms' absolute
values; over T.  Its exponential's argument adds some units of the argument, a lane's sum of n terms n u of itself, the joins a few units more.  The entropy is
lse - sum_i p_i z_i / T: scores off by e move it by at most 2 e sum_i p_i |log p_i + entropy|, and the two sums, whose terms are taken from a
reference within 2^40 of them, by their own errors times how far the terms are from that reference.  Given and likeliest items' scores by W phi are sums in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def draw_codes(N, m, b, B, n, seed, spread=3.0, wide=False):
    rng = np.random.default_rng(seed)
    codes = torch.from_numpy(rng.integers(0, b, (N, m)).astype(np.uint16 if wide else np.uint8)).cuda()
    S = torch.from_numpy((rng.standard_normal((B, m, b)) * spread / np.sqrt(m)).astype(np.float32)).cuda()
    return codes, S, torch.from_numpy(rng.integers(-2, N + 2, (B, n)).astype(np.int32)).cuda()


def draw_dense(N, d, B, n, type, seed, spread=2.5):
    rng = np.random.default_rng(seed)
    W = torch.from_numpy((rng.standard_normal((N, d)) * d ** -0.5).astype(np.float32)).to(TYPES[type]).cuda()
    H = torch.from_numpy((rng.standard_normal((B, d)) * spread).astype(np.float32)).to(TYPES[type]).cuda()
    return W, H, torch.from_numpy(rng.integers(-2, N + 2, (B, n)).astype(np.int32)).cuda()


def call(pq, first, second, *args, **kwargs):
    if first.dtype == torch.uint8:
        return pq.pq_log_probs(first, second, *args, **kwargs)
    return (pq.pq_log_probs_u16 if first.dtype == torch.uint16 else pq.pq_default_log_probs)(first, second, *args, **kwargs)


def scores(first, second):
    """Scores in 64 bits, Eq. 5's float32 chain (or None), and the largest sum of absolute values of a finite score."""
    if first.dtype in (torch.uint8, torch.uint16):
        codes = first.to(torch.int32).long()
        z64 = torch.zeros((second.shape[0], codes.shape[0]), dtype=torch.float64, device="cuda")
        size, chain = z64.clone(), None
        for k in range(codes.shape[1]):
            part = second[:, k, :][:, codes[:, k]]
            z64 += part.double()
            size += part.double().abs()
            chain = part if chain is None else chain + part
        finite = size.isfinite()
        return z64, chain + 0.0, (size[finite].max().item() if finite.any() else 0.0) * (codes.shape[1] - 1) * U, size[finite].max().item() if finite.any() else 0.0
    z64 = second.double() @ first.double().t().contiguous()
    size = (second.double().abs() @ first.double().abs().t().contiguous()).max().item()
    return z64, None, (first.shape[1] + 2) * U * size, size


def ranks(z, K):
    """The K best by score descending, then id ascending."""
    return torch.sort(z, dim=1, descending=True, stable=True).indices[:, :K].to(torch.int32)


def check(pq, first, second, items, K, T=1.0):
    N, B = first.shape[0], second.shape[0]
    got = call(pq, first, second, items, K, T)
    log_probs, entropy, lse, top_items, top_log_probs = [t.double() for t in got]
    z64, chain, off, size = scores(first, second)
    z, size, off = z64 / T, size / T, off / T + 2 * U * size / T
    want_lse = torch.logsumexp(z, 1)
    tol = off + U * (N / 512 + 64 + 4 * size + 4 * np.log(max(N, 2)))
    empty = want_lse == -np.inf
    assert torch.equal(lse[empty], want_lse[empty]) and ((lse - want_lse).abs()[~empty] <= tol).all()
    lp = torch.where(empty[:, None], -np.inf, z - want_lse[:, None])
    p = lp.exp()
    p_lp = torch.where(p > 0, p * lp, 0.0)
    want_entropy = -p_lp.sum(1)
    around = torch.where(p > 0, p * (lp + want_entropy[:, None]).abs(), 0.0).sum(1)
    tol_entropy = 2 * (off + U * (4 * size + 64)) * around + U * (N / 512 + 64) * (64 + 2 * want_entropy)
    assert ((entropy - want_entropy).abs() <= tol_entropy).all() and (entropy[empty] == 0).all()
    items = items.long()
    there = (items >= 0) & (items < N)
    want = torch.where(there, lp.gather(1, torch.where(there, items, 0)), 0.0)
    low = want == -np.inf
    assert torch.equal(log_probs[low], want[low]) and not log_probs[~there].any()
    assert ((log_probs - want).abs()[~low] <= tol + off + 2 * U * want[~low].abs()).all()
    best = ranks(chain if chain is not None else z64, K)
    assert torch.equal(got[3], best)
    want = lp.gather(1, best.long())
    low = want == -np.inf
    assert torch.equal(top_log_probs[low], want[low]) and ((top_log_probs - want).abs()[~low] <= tol + off + 2 * U * want[~low].abs()).all()
    return got


CODES = [(1, 1, 1, 1, 1, 1, False), (2, 2, 3, 1, 0, 2, False), (63, 1, 200, 3, 4, 5, False), (1000, 3, 256, 5, 1, 512, False), (4097, 4, 64, 2, 7, 0, False), (16_384, 4, 256, 1, 1, 10, False),
         (16_385, 4, 256, 1, 1, 10, False), (20_007, 8, 256, 3, 1100, 10, False), (50_003, 8, 256, 9, 3, 100, False), (70_001, 16, 256, 4, 1, 512, False), (40_001, 32, 256, 6, 1, 33, False),
         (17_500, 64, 256, 2, 1, 20, False), (17_000, 128, 256, 1, 2, 3, False), (17_900, 100, 17, 3, 1, 64, False), (100_003, 2, 256, 1, 1, 300, False), (33_333, 8, 256, 70, 2, 17, False),
         (1, 4, 300, 2, 1, 1, True), (30_049, 4, 300, 3, 2, 40, True), (20_000, 8, 1024, 5, 1, 10, True), (18_201, 16, 1024, 1, 1, 100, True), (17_600, 7, 4096, 2, 1, 7, True),
         (30_000, 2, 13, 9, 1, 5, True)]


@pytest.mark.parametrize("N,m,b,B,n,K,wide", CODES)
def test_by_sub_ids(pq, N, m, b, B, n, K, wide):
    check(pq, *draw_codes(N, m, b, B, n, seed=N + m + B, wide=wide), K)


DENSE = [(1, 8, 1, 1, 1), (2, 16, 3, 0, 2), (255, 64, 64, 3, 255), (257, 72, 128, 1, 10), (1000, 512, 1, 5, 100), (1003, 512, 50, 1, 0), (5000, 256, 129, 2, 512), (3001, 136, 300, 1, 7), (16_384, 64, 7, 1, 20),
         (16_385, 64, 7, 1, 20), (40_007, 64, 7, 70, 10), (30_003, 1032, 33, 1, 64), (60_001, 128, 257, 1, 100), (50_003, 200, 64, 1, 512), (33_001, 512, 65, 4, 33), (100_003, 512, 3, 1, 1), (70_001, 64, 1030, 1, 5)]


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("N,d,B,n,K", DENSE)
def test_by_the_default_scorer(pq, N, d, B, n, K, type):
    check(pq, *draw_dense(N, d, B, n, type, seed=N + d + B), K)


@pytest.mark.parametrize("T", [0.25, 0.7, 3.0, 100.0])
def test_temperatures(pq, T):
    check(pq, *draw_codes(30_001, 8, 256, 5, 3, seed=1), 20, T)
    for type in TYPES:
        check(pq, *draw_dense(30_001, 128, 9, 3, type, seed=2), 20, T)
        check(pq, *draw_dense(30_001, 128, 90, 3, type, seed=2), 20, T)


@pytest.mark.parametrize("kind", ["u8", "u16", "f32", "bf16", "few"])
def test_scores_in_the_worst_orders(pq, kind):
    # every later item better, then every one worse, then all alike: lists hold a piece whatever passes the floors, ties go to the lowest id
    N, K = 60_000, 50
    rise = torch.arange(N, device="cuda")
    if kind in ("u8", "u16"):
        b = 256 if kind == "u8" else 300
        S = torch.stack([torch.arange(b, device="cuda", dtype=torch.float32).repeat(1, 1) * 256, torch.arange(b, device="cuda", dtype=torch.float32).repeat(1, 1)], 1) / 4096
        codes = torch.stack([rise // 256 % 256, rise % 256], 1).to(torch.uint8 if kind == "u8" else torch.uint16)
        S = torch.cat([S, -S, torch.zeros_like(S)])
        first, second = codes, S
    else:
        # (whole numbers below 2^24 in sums of two products: exact)
        type = "bf16" if kind == "few" else kind
        W = torch.zeros((N, 64), device="cuda")
        W[:, 0], W[:, 1] = (rise // 256).float(), (rise % 256).float()
        H = torch.zeros((3 if kind != "bf16" else 99, 64), device="cuda")
        H[0, 0], H[0, 1] = 2.0 ** -4, 2.0 ** -12
        H[1] = -H[0]
        first, second = W.to(TYPES[type]), H.to(TYPES[type])
    _, _, _, top, lp = call(pq, first, second, None, K)
    want = torch.stack([rise.flip(0)[:K], rise[:K], rise[:K]]).to(torch.int32)
    assert torch.equal(top[:3], want)
    assert torch.allclose(lp[2].double(), torch.full((K,), -np.log(N), dtype=torch.float64, device="cuda"), rtol=0, atol=U * (N / 512 + 128))


@pytest.mark.parametrize("N", [45, 300, 700, 5_000, 16_000, 20_000])
@pytest.mark.parametrize("K", [1, 10, 40, 41])
@pytest.mark.parametrize("B", [2, 300])
def test_few_different_scores(pq, N, K, B):
    codes, S, items = draw_codes(N, 2, 3, B, 2, seed=N + K)
    S.copy_(S.round())                                          # (sums of them are exact)
    S[1] = 0.5
    check(pq, codes, S, items, K)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("B", [5, 100])
def test_items_twice_in_the_catalogue(pq, B, type):
    W, H, items = draw_dense(20_000, 64, B, 1, type, seed=4)
    W[10_000:] = W[:10_000]
    _, _, _, top, lp = call(pq, W, H, items, 40)
    assert torch.equal(top[:, 1::2], top[:, ::2] + 10_000) and torch.equal(lp[:, 1::2], lp[:, ::2]) and (top[:, ::2] < 10_000).all()


@pytest.mark.parametrize("wide", [False, True])
def test_sub_ids_out_of_play(pq, wide):
    codes, S, items = draw_codes(30_000, 4, 300 if wide else 256, 5, 6, seed=5, wide=wide)
    S[0, 1, 5:] = -np.inf                                       # a few hundred items are left
    S[1, 2] = -np.inf                                           # none
    S[2, 0, ::2] = -np.inf
    S[3, 3, 1:] = -np.inf                                       # about a hundred: fewer than asked for
    check(pq, codes, S, items, 200)


@pytest.mark.parametrize("N,m,b,B,wide", [(16_000, 4, 256, 5, False), (600_000, 16, 256, 110, False), (1_100_000, 8, 300, 130, True)])
def test_sub_ids_out_of_play_where_scores_go_to_lists(pq, N, m, b, B, wide):
    codes, S, items = draw_codes(N, m, b, B, 2, seed=N, wide=wide)
    S[0, 1, 5:] = -np.inf
    S[1, 2] = -np.inf
    S[2, 0, ::2] = -np.inf
    S[3, :2, 1:] = -np.inf                                      # a few items: fewer than asked for
    S[4, 0, 3] = -1e30                                          # a mask that is a number
    check(pq, codes, S, items, 60)


@pytest.mark.parametrize("N", [10_000, 30_000])
def test_a_nan_beside_sub_ids_out_of_play(pq, N):
    codes, S, items = draw_codes(N, 4, 256, 3, 2, seed=N)
    clean = call(pq, codes, S, items, 100)                       # (of as many positions: what is summed in which order goes by the shape)
    S[1, :2, 1:] = -np.inf
    S[1, 3, ::3] = float("nan")
    got = call(pq, codes, S, items, 100)
    for a, b in zip(got, clean):
        assert torch.equal(a[::2], b[::2])
    ids = got[3][1].tolist()
    assert got[2][1].isnan() and got[4][1].isnan().all() and len(set(ids)) == 100 and all(0 <= i < N for i in ids)


def test_positions_that_are_all_the_lowest_number(pq):
    codes, S, items = draw_codes(20_000, 4, 256, 3, 2, seed=5)
    S[1] = -1e30
    log_probs, entropy, lse, top, lp = call(pq, codes, S, items, 5)
    assert lse[1] == -np.inf and entropy[1] == 0 and (log_probs[1][(items[1] >= 0) & (items[1] < 20_000)] == -np.inf).all() and (lp[1] == -np.inf).all()
    assert torch.equal(top[1].cpu(), torch.arange(5, dtype=torch.int32))


@pytest.mark.parametrize("N", [9_000, 30_000])
@pytest.mark.parametrize("lowest", [-2e32, float(np.finfo(np.float32).min)])
def test_masks_of_the_lowest_number_are_masks(pq, N, lowest):
    codes, S, items = draw_codes(N, 4, 256, 3, 40, seed=7)
    S[0, 1, ::2] = lowest                                       # one masked sub-id of an item's, or two
    S[0, 2, ::2] = lowest
    S[1, 3, 1:] = lowest                                        # fewer items than asked for
    S[2] = lowest
    masked = S.clone()
    masked[S == lowest] = -np.inf
    for got, want in zip(call(pq, codes, S, items, 200), call(pq, codes, masked, items, 200)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("odd", [float("nan"), float("inf")])
@pytest.mark.parametrize("kind", ["u8", "f32", "bf16", "f16", "many"])
def test_scores_that_are_no_numbers_stay_with_their_position(pq, kind, odd):
    N, K = 30_000, 20
    if kind == "u8":
        first, second, items = draw_codes(N, 4, 256, 5, 3, seed=6)
        bad = second.clone()
        bad[2, 1, 7] = odd
    else:
        first, second, items = draw_dense(N, 64, 70 if kind == "many" else 5, 3, "bf16" if kind == "many" else kind, seed=6)
        bad = second.clone()
        bad[2, 7] = odd
    clean, got = call(pq, first, second, items, K), call(pq, first, bad, items, K)
    rest = [q for q in range(second.shape[0]) if q != 2]
    for a, b in zip(clean, got):
        assert torch.equal(a[rest], b[rest])
    named = (items[2] >= 0) & (items[2] < N)
    assert got[0][2][named].isnan().all() and got[1][2].isnan() and got[2][2].isnan() and got[4][2].isnan().all()
    ids = got[3][2].tolist()
    assert len(set(ids)) == K and all(0 <= i < N for i in ids)


def test_alternatives_are_those_of_the_ranking(pq):
    codes, S, _ = draw_codes(300_001, 8, 256, 33, 1, seed=7)
    ids, ranked = pq.pq_score_topk(codes, S, 100)
    _, _, lse, top, lp = pq.pq_log_probs(codes, S, None, 100)
    assert torch.equal(ids, top)
    # the log-sum that they are made with has 64 bits: the one returned is off by its rounding, U |lse|, and they are rounded themselves
    assert ((lp.double() - (ranked.double() - lse.double()[:, None])).abs() <= U * (lp.abs() + lse.abs()[:, None])).all()


def test_given_items_are_those_of_the_loss(pq):
    codes, S, items = draw_codes(50_001, 8, 256, 33, 1, seed=8)
    loss, lse = pq.pq_cross_entropy(codes, S, items[:, 0].contiguous())
    log_probs, _, lse2, _, _ = pq.pq_log_probs(codes, S, items)
    size = S.abs().amax(2).sum(1).max().item()
    tol = 2 * U * (8 * size + 50_001 / 512 + 128 + 4 * size)
    assert ((loss + log_probs[:, 0]).abs() <= tol).all() and ((lse - lse2).abs() <= tol).all()


@pytest.mark.parametrize("kind", ["u8", "bf16", "many"])
def test_same_bits_every_time_and_on_any_stream(pq, kind):
    first, second, items = draw_codes(200_003, 8, 256, 9, 3, seed=9) if kind == "u8" else draw_dense(200_003, 64, 300 if kind == "many" else 9, 3, "bf16", seed=9)
    want = call(pq, first, second, items, 100)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [call(pq, first, second, items, 100) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    for got in again:
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("kind", ["u8", "f32", "bf16", "many"])
def test_in_a_graph(pq, kind):
    N, K = 50_001, 20

    def inputs(seed):
        return draw_codes(N, 4, 256, 5, 2, seed) if kind == "u8" else draw_dense(N, 64, 130 if kind == "many" else 5, 2, "f32" if kind == "f32" else "bf16", seed)

    first, second, items = inputs(1)
    outputs = [t.clone() for t in call(pq, first, second, items, K)]
    workspace = torch.empty(pq.pq_log_probs_workspace_bytes(N, 5, 4, 256, K) if kind == "u8"
                            else pq.pq_default_log_probs_workspace_bytes(N, second.shape[0], 64, 0 if kind == "f32" else 1, K), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(pq, first, second, items, K, 1.0, workspace, *outputs)
    for seed in (2, 3, 4):
        for to, new in zip((first, second, items), inputs(seed)):
            to.copy_(new)
        workspace.random_(0, 256)
        want = [t.clone() for t in call(pq, first, second, items, K)]
        for t in outputs:
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outputs))


def test_a_workspace_as_large_as_said_and_no_larger(pq):
    for N, B, K in ((40_000, 70, 100), (10_000, 3, 10), (17_000, 1, 512)):
        for type, code in (("f32", 0), ("bf16", 1)):
            W, H, items = draw_dense(N, 64, B, 2, type, seed=B)
            need = pq.pq_default_log_probs_workspace_bytes(N, B, 64, code, K)
            room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
            want = call(pq, W, H, items, K)
            got = call(pq, W, H, items, K, 1.0, room[:need])
            assert (room[need:] == 0xA5).all() and all(torch.equal(a, b) for a, b in zip(want, got))
        codes, S, items = draw_codes(N, 4, 256, B, 2, seed=B)
        need = pq.pq_log_probs_workspace_bytes(N, B, 4, 256, K)
        room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        want = call(pq, codes, S, items, K)
        got = call(pq, codes, S, items, K, 1.0, room[:need])
        assert (room[need:] == 0xA5).all() and all(torch.equal(a, b) for a, b in zip(want, got))


def test_rows_beyond_32_bits_of_offset(pq):
    N, d, B = 4_300_000, 512, 2                                  # 4.4 GB of W
    W = torch.zeros((N, d), dtype=torch.bfloat16, device="cuda")
    H = torch.zeros((B, d), dtype=torch.bfloat16, device="cuda")
    H[:, 0] = 1.0
    marked = torch.tensor([N - 1, 4_200_001, 17, 3_000_000], device="cuda")
    W[marked, 0] = torch.tensor([20.0, 18.0, 16.0, 14.0], device="cuda").bfloat16()
    log_probs, entropy, lse, top, lp = pq.pq_default_log_probs(W, H, marked.to(torch.int32).repeat(B, 1).contiguous(), 4)
    assert torch.equal(top.long(), marked.repeat(B, 1)) and torch.equal(lp, log_probs)
    want = torch.logsumexp(torch.cat([W[marked, 0].double(), torch.full((1,), np.log(N - 4), dtype=torch.float64, device="cuda")]), 0)
    assert ((lse.double() - want).abs() <= U * (N / 512 + 64 + 80)).all()
    del W, H
    torch.cuda.empty_cache()


def test_refusals(pq):
    codes, S, items = draw_codes(500, 4, 256, 3, 2, seed=1)
    W, H, _ = draw_dense(500, 64, 3, 2, "bf16", seed=1)
    for first, second in ((codes, S), (W, H)):
        for bad in (dict(K=-1), dict(K=501), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan"))):
            with pytest.raises(pq.PQError) as e:
                call(pq, first, second, items, **bad)
            assert e.value.code == pq.PQ_ERR_SHAPE, bad
        for bad in (dict(temperature=1e-5), dict(temperature=1e5), dict(temperature=float("inf"))):
            with pytest.raises(pq.PQError) as e:
                call(pq, first, second, items, **bad)
            assert e.value.code == pq.PQ_ERR_UNSUPPORTED, bad
        with pytest.raises(pq.PQError) as e:
            call(pq, first, second, items, 10, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
        assert e.value.code == pq.PQ_ERR_WORKSPACE
        for bad in (items.long(), items[:2], items[0], items.t(), items.cpu()):
            with pytest.raises(ValueError):
                call(pq, first, second, bad, 5)
        with pytest.raises(ValueError):
            call(pq, first, second, items, 5, top_items=torch.empty((3, 4), dtype=torch.int32, device="cuda"))
        with pytest.raises(ValueError):
            call(pq, first, second.cpu(), items, 5)
    big, H2, _ = draw_dense(600, 64, 3, 2, "bf16", seed=1)
    with pytest.raises(pq.PQError) as e:
        call(pq, big, H2, items, 513)
    assert e.value.code == pq.PQ_ERR_UNSUPPORTED
    with pytest.raises(ValueError):
        pq.pq_default_log_probs(W.double(), H.double(), items)
    with pytest.raises(pq.PQError):
        pq.pq_default_log_probs(W, H[:, :32].contiguous(), items)


def test_by_lists_of_sub_ids_again_and_in_a_graph(pq):
    N, m, B, K = 50_001, 32, 40, 30                             # (more lookups than the ranking is asked for: pieces, cuts, lists)
    codes, S, items = draw_codes(N, m, 256, B, 2, seed=1)
    want = [t.clone() for t in check(pq, codes, S, items, K)]
    outputs = [t.clone() for t in want]
    workspace = torch.empty(pq.pq_log_probs_workspace_bytes(N, B, m, 256, K), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(pq, codes, S, items, K, 1.0, workspace, *outputs)
    for seed in (1, 2, 3):
        for to, new in zip((codes, S, items), draw_codes(N, m, 256, B, 2, seed)):
            to.copy_(new)
        workspace.random_(0, 256)
        if seed > 1:
            want = [t.clone() for t in call(pq, codes, S, items, K)]
        for t in outputs:
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outputs))


@pytest.mark.parametrize("kind", ["u8", "lists", "f32", "bf16", "many"])
def test_two_calls_at_once(pq, kind):
    def inputs(seed):
        if kind in ("u8", "lists"):
            return draw_codes(60_001, 32 if kind == "lists" else 4, 256, 40, 3, seed=seed)
        return draw_dense(60_001, 64, 200 if kind == "many" else 9, 3, "f32" if kind == "f32" else "bf16", seed=seed)

    both = [inputs(1), inputs(2)]
    want = [call(pq, *each, 20) for each in both]
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, side in enumerate(sides):
            with torch.cuda.stream(side):
                got[i].append(call(pq, *both[i], 20))
    torch.cuda.synchronize()
    for i in range(2):
        for each in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(want[i], each))


@pytest.mark.parametrize("kind", ["u8", "f32", "bf16", "many"])
def test_entropy_alone(pq, kind):
    first, second, _ = draw_codes(30_001, 4, 256, 5, 1, seed=3) if kind == "u8" else draw_dense(30_001, 64, 130 if kind == "many" else 5, 1, "f32" if kind == "f32" else "bf16", seed=3)
    log_probs, entropy, lse, top_items, top_log_probs = call(pq, first, second)
    B = second.shape[0]
    assert log_probs.shape == top_items.shape == top_log_probs.shape == (B, 0)
    check(pq, first, second, torch.empty((B, 0), dtype=torch.int32, device="cuda"), 0)


@pytest.mark.parametrize("B", [3, 300])
@pytest.mark.parametrize("type", list(TYPES))
def test_as_many_likeliest_items_as_can_be_asked_for(pq, type, B):
    check(pq, *draw_dense(513 if B == 3 else 9_001, 24, B, 2, type, seed=B), 512)


@pytest.mark.parametrize("B", [1, 5, 100, 300])
@pytest.mark.parametrize("type", list(TYPES))
def test_items_that_the_catalogue_holds_hundreds_of_times(pq, type, B):
    W, H, items = draw_dense(130, 96, B, 2, type, seed=B)
    N = 60_001
    W = W[torch.from_numpy(np.random.default_rng(4).integers(0, 130, N)).cuda()].contiguous()
    z64 = H.double() @ W.double().t().contiguous()
    assert torch.equal(call(pq, W, H, items, 20)[3], ranks(z64, 20))      # (of as good ones the lowest ids: equal rows have equal sums wherever they are)
