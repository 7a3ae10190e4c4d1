"""Corners of the log-probabilities and the distillation: tables that fill LDS, masks that are numbers, low temperatures, lists
that are kept to their size.

Bounds are those of test_log_probs_gpu.py, but of every position by its own scores, and by those alone that do not count as -inf."""
import numpy as np
import pytest
import torch

import test_distillation_gpu as teaching
import test_log_probs_gpu as probs

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LEAST = -(2.0 ** 23 + 126) * np.log(2.0)                        # scores over T below it count as -inf


def check_by_position(pq, first, second, items, K, T=1.0, rows=None):
    N = first.shape[0]
    got = probs.call(pq, first, second, items, K, T)
    if rows is not None:                                        # (of many positions these are looked at)
        got, second, items = [t[rows] for t in got], second[rows], items[rows]
    log_probs, entropy, lse, _, top_log_probs = [t.double() for t in got]
    z64, chain, _, _ = probs.scores(first, second)
    if chain is None:
        terms, additions = second.double().abs() @ first.double().abs().t().contiguous(), first.shape[1] + 2
    else:
        codes = first.to(torch.int32).long()
        terms, additions = sum(second[:, k, :][:, codes[:, k]].double().abs() for k in range(codes.shape[1])), codes.shape[1] - 1
    play = z64 / T >= LEAST
    z = torch.where(play, z64 / T, -np.inf)
    size = torch.where(play, terms, 0.0).amax(1) / T
    off = (additions + 2) * U * size
    tol = off + U * (N / 512 + 64 + 4 * size + 4 * np.log(max(N, 2)))
    want_lse = torch.logsumexp(z, 1)
    empty = want_lse == -np.inf
    assert torch.equal(lse[empty], want_lse[empty]) and ((lse - want_lse).abs() <= tol)[~empty].all()
    lp = torch.where(empty[:, None], -np.inf, z - want_lse[:, None])
    p_lp = torch.where(lp > -np.inf, lp.exp() * lp, 0.0)
    want = -p_lp.sum(1)
    around = torch.where(lp > -np.inf, lp.exp() * (lp + want[:, None]).abs(), 0.0).sum(1)
    assert ((entropy - want).abs() <= 2 * (off + U * (4 * size + 64)) * around + U * (N / 512 + 64) * (64 + 2 * want)).all() and not entropy[empty].any()
    there = (items >= 0) & (items < N)
    best = probs.ranks(chain if chain is not None else z64, K)
    assert torch.equal(got[3], best)
    for out, want in ((log_probs, torch.where(there, lp.gather(1, torch.where(there, items, 0).long()), 0.0)), (top_log_probs, lp.gather(1, best.long()))):
        low = want == -np.inf
        assert torch.equal(out == -np.inf, low)
        assert ((out - want).abs() <= (tol + off)[:, None] + 2 * U * want.abs())[~low].all()
    return got


@pytest.mark.parametrize("m,b,B", [(4, 2544, 3), (8, 1272, 5), (16, 636, 3), (8, 2544, 2), (1, 20352, 3), (8, 1271, 3)])
def test_tables_as_large_as_lds(pq, m, b, B):
    # (Q queries' tables of m b floats and the sums of the waves fill 160 KB to the last 16 bytes)
    probs.check(pq, *probs.draw_codes(20_001, m, b, B, 3, seed=m + b, wide=True), 10)
    probs.check(pq, *probs.draw_codes(3_001, m, b, B, 3, seed=m + b, wide=True), 10)


@pytest.mark.parametrize("mask", [-1e30, -1e9, -6e6])
@pytest.mark.parametrize("N,m,b,B,wide", [(9_000, 4, 256, 5, False), (30_000, 4, 256, 5, False), (30_000, 32, 256, 40, False), (20_000, 4, 300, 3, True)])
def test_sub_ids_masked_by_a_number(pq, N, m, b, B, wide, mask):
    codes, S, items = probs.draw_codes(N, m, b, B, 40, seed=N + m, wide=wide)
    S[0, 1, ::2] = mask
    S[1, 0, 1:] = mask                                          # about a hundred items are left: fewer than asked for
    S[2] = mask                                                 # none
    check_by_position(pq, codes, S, items, 300)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B", [5, 130])
def test_items_masked_by_a_number(pq, B, type):
    N = 20_000
    W, H, items = probs.draw_dense(N, 64, B, 40, type, seed=B)
    W[:, 0], H[:, 0] = 0.0, 0.0
    W[::3, 0], H[1, 0] = (-60_000.0, 60_000.0) if type == "f16" else (-1e30, 1.0)
    check_by_position(pq, W, H, items, 50)


def test_scores_at_the_border_of_what_counts(pq):
    # one split, whose entries are the scores: whether an item counts is the same for its log-probability and for the log-sum of a position that has no other
    border = 2.0 ** 23 * np.log(2.0)
    S = torch.tensor([[-1.0, -border + 1, -border - 1, -border - 200, -1e30, 0.5], [-border + 1] * 6, [-border - 200] * 6], dtype=torch.float32, device="cuda")[:, None, :].contiguous()
    codes = torch.arange(6, dtype=torch.uint8, device="cuda")[:, None].contiguous()
    items = torch.arange(6, dtype=torch.int32, device="cuda").repeat(3, 1)
    log_probs, _, lse, _, _ = pq.pq_log_probs(codes, S, items)
    counts = torch.tensor([[True, True, True, False, False, True], [True] * 6, [False] * 6], device="cuda")
    assert torch.equal(log_probs > -np.inf, counts) and torch.equal(lse > -np.inf, counts.any(1))


@pytest.mark.parametrize("T", [0.5, 2.0])
def test_listed_items_masked_by_a_number(pq, T):
    codes, S, items, scores, grad = teaching.draw_codes(3_000, 4, 256, 5, 8, seed=5)
    S[1, 2] = -1e30                                             # nothing is left: no loss, no gradient
    S[2, 0, ::2] = -1e30                                        # listed items among those out of play: the loss is infinite, the gradient is not
    masked = torch.where(S == -1e30, -np.inf, S)
    for step in (teaching.forward, lambda *a: (teaching.backward(*a[:5], lse, grad, T),)):
        got, want = step(pq, codes, S, items, scores, T), step(pq, codes, masked, items, scores, T)
        lse = got[-1]
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    loss, lse = teaching.forward(pq, codes, S, items, scores, T)
    dS = teaching.backward(pq, codes, S, items, scores, lse, grad, T)
    assert loss[1] == 0 and loss[2] == np.inf and loss[[0, 3, 4]].isfinite().all() and not dS[1].any() and dS.isfinite().all()
    for type in ("f32", "bf16"):
        for B in (5, 90):
            W, H, items, scores, grad = teaching.draw_dense(3_000, 64, B, 8, type, seed=6)
            W[:, 0], H[:, 0] = 0.0, 0.0
            W[::2, 0], H[2, 0] = -1e30, 1.0
            items[2] = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7], device="cuda")
            loss, lse = teaching.forward(pq, W, H, items, scores, T)
            rest = torch.arange(B, device="cuda") != 2
            assert loss[2] == np.inf and loss[rest].isfinite().all() and lse.isfinite().all()


@pytest.mark.parametrize("T", [0.01, 0.07, 0.3, 3.0])
@pytest.mark.parametrize("kind", ["u8", "lists", "u16", "f32", "bf16", "many"])
def test_log_probabilities_of_large_scores_at_low_temperatures(pq, kind, T):
    # One item of the score 20, and in position 1 a second one that is half as likely, all others 0 or below.  The sums' reference c is the largest score times log2 e / T as float32
    # numbers, and what the item's own exponent is off it is kept (fma): its exponential is 2^x, |x| <= 2^-24 c, off by a unit (2 u), of which the others, below 2^-20 of it, take at most
    # 2^-20 N; a second one adds as much and a rounding, in joins (some 40, of which one adds them and the others add nothing).  So log p is off by some 16 u; that the log-sum and
    # its score were made by two factors log2 e / T, one of them rounded, would be up to 2^-24 of 20 / T.
    N, B = 30_000, 200 if kind == "many" else 40 if kind == "lists" else 3
    second = float(np.float32(20.0) - np.float32(T) * np.float32(np.log(2.0)))
    if kind in ("f32", "bf16", "many"):
        W, H = torch.zeros((N, 64), device="cuda"), torch.zeros((B, 64), device="cuda")
        W[17, 0], W[29_999, 1], H[:, 0] = 4.0, 1.0, 5.0
        H[1, 1] = second
        type = torch.float32 if kind == "f32" else torch.bfloat16
        first, queries = W.to(type), H.to(type)
        z = queries.double() @ first.double().t().contiguous()
    else:
        m = 32 if kind == "lists" else 4
        first = torch.full((N, m), 3, dtype=torch.uint8 if kind != "u16" else torch.uint16, device="cuda")
        first.view(torch.uint8 if kind != "u16" else torch.int16)[17, 1] = 5
        first.view(torch.uint8 if kind != "u16" else torch.int16)[29_999, 2] = 7
        queries = torch.zeros((B, m, 300 if kind == "u16" else 256), device="cuda")
        queries[:, 1, 5] = 20.0
        queries[1, 2, 7] = second
        z = torch.zeros((B, N), dtype=torch.float64, device="cuda")
        z[:, 17] = 20.0
        z[1, 29_999] = second
    T32 = float(np.float32(T))
    items = torch.tensor([17, 29_999], dtype=torch.int32, device="cuda").repeat(B, 1)
    log_probs, _, lse, top, top_log_probs = probs.call(pq, first, queries, items, 2, T)
    want_lse = torch.logsumexp(z / T32, 1)
    want = (z / T32 - want_lse[:, None])[:, [17, 29_999]]
    assert (log_probs <= 0).all() and (top_log_probs <= 0).all() and (top[:, 0] == 17).all() and torch.equal(top_log_probs[:, 0], log_probs[:, 0])
    exact = 16 * U + (0 if T < 1 else 64 * U)                    # (at T = 3 the other items have most of the mass: N / 512 additions of a lane more)
    assert ((log_probs.double() - want).abs() <= exact + U * want.abs()).all()
    assert ((lse.double() - want_lse).abs() <= exact + U * want_lse.abs()).all()


@pytest.mark.parametrize("N,B,K", [(16_384, 20_000, 10), (12_000, 65_535, 3), (270_001, 65_535, 5)])
def test_lists_that_are_kept_to_their_size(pq, N, B, K):
    # catalogues that one piece would hold, but for so many positions; and pieces whose sums take the places of those before
    rows = torch.randint(0, B, (40,), generator=torch.Generator().manual_seed(N)).cuda()
    rows[0], rows[1] = 0, B - 1
    check_by_position(pq, *probs.draw_codes(N, 4, 64, B, 2, seed=N), K, rows=rows)
    for type in ("f32", "bf16"):
        check_by_position(pq, *probs.draw_dense(N, 8, B, 2, type, seed=B), K, rows=rows)
    torch.cuda.empty_cache()


def test_sums_of_many_pieces_of_few_positions(pq):
    # 286 pieces of 2^28 / 64 items, whose sums of 256 groups share their places.  All scores but four are 0: every lane's sum is a whole number
    N, B = 1_200_000_000, 64
    W, H = torch.zeros((N, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros((B, 8), dtype=torch.bfloat16, device="cuda")
    H[:, 0] = 1.0
    marked = torch.tensor([N - 1, 1_100_000_001, 17, 300_000_000], device="cuda")
    W[marked, 0] = torch.tensor([20.0, 18.0, 16.0, 14.0], device="cuda").bfloat16()
    assert pq.pq_default_log_probs_workspace_bytes(N, B, 8, 1, 4) < 2 ** 31 + 2 ** 25
    log_probs, entropy, lse, top, lp = pq.pq_default_log_probs(W, H, marked.to(torch.int32).repeat(B, 1).contiguous(), 4)
    assert torch.equal(top.long(), marked.repeat(B, 1)) and torch.equal(lp, log_probs)
    z = torch.cat([W[marked, 0].double(), torch.zeros(1, dtype=torch.float64, device="cuda")])
    count = torch.tensor([1.0, 1.0, 1.0, 1.0, N - 4.0], dtype=torch.float64, device="cuda")
    want = torch.log((count * z.exp()).sum())
    p = (z - want).exp()
    # a join adds 4 u of a sum; a position's sums meet in some 300
    assert ((lse.double() - want).abs() <= 1200 * U).all() and ((entropy.double() - (count * p * (want - z)).sum()).abs() <= 1200 * U * 64).all()
    del W
    torch.cuda.empty_cache()


@pytest.mark.parametrize("K", [1, 40, 100, 512])
@pytest.mark.parametrize("N,m,b,B", [(60_000, 8, 256, 330), (60_000, 4, 256, 1_300), (60_000, 32, 256, 100), (60_000, 16, 300, 400), (60_000, 4, 300, 1_300)])
def test_lists_of_sub_ids_in_the_worst_orders(pq, N, m, b, B, K):
    # (more lookups than the ranking is asked for, N B m^2 over 1.2e9, or over 6e9: pieces, floors, regions.)  Every third position's later items are all better, so that whatever a
    # region has room for comes to it, every third's are worse, and every third's are alike: sums of whole numbers over 4096 are exact, ties go to the lowest id
    assert N * B * m * m > (1.2e9 if K <= 40 or B >= 128 else 6e9)
    rise = torch.arange(N, device="cuda")
    digits = torch.stack([rise // 256, rise % 256], 1)
    codes = torch.cat([digits, torch.full((N, m - 2), 9, device="cuda")], 1).to(torch.uint8 if b == 256 else torch.uint16).contiguous()
    S = torch.zeros((B, m, b), device="cuda")
    S[:, 0, :256], S[:, 1, :256] = torch.arange(256, device="cuda") / 16, torch.arange(256, device="cuda") / 4096
    S[1::3] *= -1
    S[2::3] = 0.0
    _, _, lse, top, lp = probs.call(pq, codes, S, None, K)
    assert (top[::3] == rise.flip(0)[:K]).all() and (top[1::3] == rise[:K]).all() and (top[2::3] == rise[:K]).all()
    z = rise.double() / 4096
    for q, x in ((0, z), (1, -z), (2, 0 * z)):
        want = torch.logsumexp(x, 0)
        tol = U * (N / 512 + 64 + 4 * 15 + 4 * np.log(N)) + 2 * U * 15
        assert ((lse[q::3].double() - want).abs() <= tol).all()
        assert ((lp[q::3].double() - (x[top[q].long()] - want)).abs() <= tol + 2 * U * 30).all()


@pytest.mark.parametrize("K", [5, 100, 512])
@pytest.mark.parametrize("type,N,d", [("bf16", 60_000, 64), ("f16", 200_000, 64), ("f16", 200_000, 136), ("bf16", 60_000, 304)])
def test_more_candidates_of_few_positions_than_wait(pq, type, N, d, K):
    # 64 positions whose later items are all better: every score passes its floor, thousands of them a workgroup, of which 1024 wait in LDS and the others go to memory at once
    B = 64
    rise = torch.arange(N, device="cuda")
    W, H = torch.zeros((N, d), device="cuda"), torch.zeros((B, d), device="cuda")
    W[:, 0], W[:, 1] = (rise // 256).float(), (rise % 256).float()
    H[:, 0], H[:, 1] = 2.0 ** -4, 2.0 ** -12
    H[1::4] *= -1
    _, _, lse, top, lp = probs.call(pq, W.to(probs.TYPES[type]), H.to(probs.TYPES[type]), None, K)
    up = torch.ones(B, dtype=torch.bool, device="cuda")
    up[1::4] = False
    assert (top[up] == rise.flip(0)[:K]).all() and (top[~up] == rise[:K]).all()
    z = rise.double() / 4096
    size = N / 4096
    tol = U * (N / 512 + 64 + 4 * size + 4 * np.log(N)) + 2 * U * size
    assert ((lse[up].double() - torch.logsumexp(z, 0)).abs() <= tol).all() and ((lse[~up].double() - torch.logsumexp(-z, 0)).abs() <= tol).all()
    assert ((lp[up].double() - (z.flip(0)[:K] - torch.logsumexp(z, 0))).abs() <= tol + 2 * U * size).all()


@pytest.mark.parametrize("N,m,b,B,K,wide", [(600_000, 16, 256, 110, 60, False), (1_100_000, 8, 300, 130, 60, True), (1_271_638, 8, 256, 64, 20, False), (1_271_638, 4, 256, 64, 40, False),
                                            (90_001, 8, 256, 300, 100, False)])
def test_lists_of_sub_ids_beside_masks(pq, N, m, b, B, K, wide):
    assert N * B * m * m > (1.2e9 if K <= 40 or B >= 128 else 6e9)
    codes, S, items = probs.draw_codes(N, m, b, B, 2, seed=N + m, wide=wide)
    check_by_position(pq, codes, S, items, K)
    S[0, 1, 5:] = -np.inf
    S[1, 2] = -np.inf                                           # none is left
    S[2, 0, ::2] = -np.inf
    S[3, :2, 1:] = -np.inf                                      # a few items: fewer than asked for
    S[4, 0, 3] = -1e30                                          # masks that are numbers
    S[5, :2, 1:] = -1e9
    S[6] = float(np.finfo(np.float32).min)
    check_by_position(pq, codes, S, items, K)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
def test_gradients_of_log_probabilities_are_a_distillations(pq, T):
    # sum_qk g_qk log p_{q,i_qk} by pq_log_probs, and its gradient by the distillation from a list of these items, as the header has it, against the definition's in 64 bits
    N, B = 3_001, 6
    g = torch.from_numpy(np.random.default_rng(1).uniform(0.1, 2.0, (B, 3)).astype(np.float32)).cuda()
    for n in (1, 3):
        scores = T * g[:, :n].double().log() if n > 1 else torch.zeros((B, 1), device="cuda")
        for first, second in (probs.draw_codes(N, 4, 256, B, 1, seed=2)[:2], probs.draw_dense(N, 64, B, 1, "f32", seed=2)[:2]):
            items = torch.from_numpy(np.stack([np.random.default_rng(q).permutation(N)[:n] for q in range(B)]).astype(np.int32)).cuda()
            leaf = second.double().requires_grad_()
            if first.dtype == torch.uint8:
                z = sum(leaf[:, k, :][:, first[:, k].long()] for k in range(4))
                size = sum(second[:, k, :].abs().amax(1) for k in range(4)).max().item()
            else:
                z = leaf @ first.double().t().contiguous()
                size = (second.double().abs() @ first.double().abs().t().contiguous()).max().item()
            lp = torch.log_softmax(z / T, 1).gather(1, items.long())
            objective = (g[:, :n].double() * lp).sum()
            want, = torch.autograd.grad(objective, leaf)
            _, lse = teaching.forward(pq, first, second, items, scores.float(), T)
            out = teaching.backward(pq, first, second, items, scores.float(), lse, -g[:, :n].sum(1) / T ** 2, T)
            out = out if first.dtype == torch.uint8 else out[0]
            ours = (g[:, :n] * probs.call(pq, first, second, items, 0, T)[0]).sum()
            # a probability is off by what its score, over T, and the log-sum are: (d + 2 + 4) u size / T and the sums' rounding; a gradient's entry adds such
            # probabilities, g of them together at most, of either sign, times (by W phi) elements of W below 1
            rel = U * ((2 * 66 + 8) * size / T + N / 512 + 200)
            assert ((out.double() - want).abs() <= 4 * g.sum(1).max().item() / T * rel).all()
            assert abs(ours.item() - objective.item()) <= g.sum().item() * 2 * rel


@pytest.mark.parametrize("B", [3, 100, 300])
def test_near_copies_are_ranked_in_64_bits(pq, B):
    # K + 16 items whose scores differ by 2^-34 of themselves, far less than a float32 sum tells apart
    N, K = 20_000, 10
    W, H, items = probs.draw_dense(N, 64, B, 1, "f32", seed=B)
    at = torch.from_numpy(np.random.default_rng(5).permutation(N)[:K + 16]).cuda()
    W[:, 62], W[:, 63], H[:, 62], H[:, 63] = 0.0, 0.0, 1.0, 1.0
    W[at] = 0.0
    W[at, 62] = 40.0
    W[at, 63] = 2.0 ** -29 * torch.arange(K + 16, device="cuda").float()
    z64 = H.double() @ W.double().t().contiguous()
    assert (z64.amax(1) < 41).all()
    top = probs.call(pq, W, H, items, K)[3]
    assert torch.equal(top.long(), at.flip(0)[:K].repeat(B, 1))
