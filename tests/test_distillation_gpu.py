"""Distillation from a teacher's list, by sub-ids and by W phi, and its gradients, against the definitions in 64 bits on the same inputs.

Bounds are those of the cross entropy's tests: u = 2^-24; a score is off by (m - 1) u or (d + 2) u times the sum of its terms' absolute values, over T; log-sum and
probabilities carry that and their sums' errors.  The teacher's weights and the loss's sum over the list are 64-bit numbers, so the loss is T^2 times
the log-sum's error and the listed scores' away (by W phi these are 64-bit sums), and rounded once."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": (torch.float32, U), "bf16": (torch.bfloat16, 2.0 ** -8), "f16": (torch.float16, 2.0 ** -11)}


def draw_teacher(rng, N, B, K):
    items = rng.integers(0, N, (B, K)).astype(np.int32)
    length = rng.integers(0, K + 1, B)
    length[::2] = K
    items[np.arange(K)[None, :] >= length[:, None]] = -1
    if K > 2:
        items[:, 2] = np.where(items[:, 2] >= 0, items[:, 0], -1)               # an item listed twice
    if K > 4:
        items[0, 4] = N                                          # no item either
    scores = (rng.standard_normal((B, K)) * 2.0 + 3.0).astype(np.float32)
    if K > 5:
        scores[0, 3] = -np.inf
    return [torch.from_numpy(a).cuda() for a in (items, scores, rng.standard_normal(B).astype(np.float32))]


def draw_codes(N, m, b, B, K, seed, spread=3.0, wide=False):
    rng = np.random.default_rng(seed)
    codes = torch.from_numpy(rng.integers(0, b, (N, m)).astype(np.uint16 if wide else np.uint8)).cuda()
    S = torch.from_numpy((rng.standard_normal((B, m, b)) * spread / np.sqrt(m)).astype(np.float32)).cuda()
    return (codes, S, *draw_teacher(rng, N, B, K))


def draw_dense(N, d, B, K, type, seed, spread=2.5):
    rng = np.random.default_rng(seed)
    W = torch.from_numpy((rng.standard_normal((N, d)) * d ** -0.5).astype(np.float32)).to(TYPES[type][0]).cuda()
    H = torch.from_numpy((rng.standard_normal((B, d)) * spread).astype(np.float32)).to(TYPES[type][0]).cuda()
    return (W, H, *draw_teacher(rng, N, B, K))


def forward(pq, first, second, *args, **kwargs):
    if first.dtype == torch.uint8:
        return pq.pq_distillation(first, second, *args, **kwargs)
    return (pq.pq_distillation_u16 if first.dtype == torch.uint16 else pq.pq_default_distillation)(first, second, *args, **kwargs)


def backward(pq, first, second, *args, **kwargs):
    if first.dtype == torch.uint8:
        return pq.pq_distillation_backward(first, second, *args, **kwargs)
    return (pq.pq_distillation_u16_backward if first.dtype == torch.uint16 else pq.pq_default_distillation_backward)(first, second, *args, **kwargs)


def weights_of(items, scores, N, T):
    """Weight and its logarithm of every entry [B][K], and whether a list has any."""
    there = (items >= 0) & (items < N)
    u = torch.where(there, scores.double() / T, -np.inf)
    any = (u > -np.inf).any(1)
    log_w = torch.where(any[:, None], u - torch.logsumexp(u, 1, keepdim=True), -np.inf)
    return log_w.exp(), log_w, any


def scores_of(first, second):
    if first.dtype in (torch.uint8, torch.uint16):
        codes = first.to(torch.int32).long()
        z = torch.zeros((second.shape[0], codes.shape[0]), dtype=torch.float64, device="cuda")
        size = z.clone()
        for k in range(codes.shape[1]):
            part = second[:, k, :][:, codes[:, k]].double()
            z += part
            size += part.abs()
        finite = size.isfinite()
        size = size[finite].max().item() if finite.any() else 0.0
        return z, size, (codes.shape[1] - 1) * U * size
    z = second.double() @ first.double().t().contiguous()
    size = (second.double().abs() @ first.double().abs().t().contiguous()).max().item()
    return z, size, (first.shape[1] + 2) * U * size


def check(pq, first, second, items, scores, grad, T=1.0, type=None):
    N, B = first.shape[0], second.shape[0]
    loss, lse = forward(pq, first, second, items, scores, T)
    got = backward(pq, first, second, items, scores, lse, grad, T)
    z, size, off = scores_of(first, second)
    z, size, off = z / T, size / T, off / T + 2 * U * size / T
    want_lse = torch.logsumexp(z, 1)
    empty = want_lse == -np.inf
    tol_lse = off + U * (N / 512 + 64 + 4 * size + 4 * np.log(max(N, 2)))
    assert torch.equal(lse[empty].double(), want_lse[empty]) and ((lse.double() - want_lse).abs()[~empty] <= tol_lse).all()
    w, log_w, any = weights_of(items, scores, N, T)
    any &= ~empty
    at = torch.where((items >= 0) & (items < N), items, 0).long()
    lp = z.gather(1, at) - torch.where(empty, 0.0, want_lse)[:, None]
    want = T * T * torch.where((w > 0) & any[:, None], w * (log_w - lp), 0.0).sum(1)
    endless = want == np.inf
    assert torch.equal(loss[endless].double(), want[endless])
    assert ((loss.double() - want).abs()[~endless] <= T * T * (tol_lse + off) + U * want[~endless].abs() + 1e-40).all()
    assert not loss[~any].any()
    p = torch.where(any[:, None], torch.exp(z - torch.where(empty, 0.0, want_lse)[:, None]), 0.0)
    dz = p.clone()
    rows = torch.arange(B, device="cuda")[:, None].expand_as(at)
    dz.index_put_((rows, at), torch.where(any[:, None], -w, 0.0), accumulate=True)
    g = torch.where(any, grad.double() * T, 0.0)
    rel = off + tol_lse + U * (4 * size + 64)                    # of a probability
    if type is None:
        codes, (m, b) = first.to(torch.int32).long(), second.shape[1:]
        assert not got[~any].any()
        for k in range(m):
            mass, want = (torch.zeros((B, b), dtype=torch.float64, device="cuda").index_add_(1, codes[:, k], x) for x in (p, dz))
            tol = g.abs()[:, None] * (mass * rel + (N + w.shape[1]) * 2.0 ** -62 + 4 * U * want.abs()) + 1e-44
            assert ((got[:, k].double() - g[:, None] * want).abs() <= tol).all()
        return loss, lse, got
    unit = TYPES[type][1]
    dz *= g[:, None]
    dH, dW = got
    dz_off = g.abs()[:, None] * p * rel + dz.abs() * (unit + 4 * U) + (2.0 ** -40 * g.abs().max() if type == "f16" else 0.0) + 1e-40
    for out, other, n, by_rows in ((dH, first.double(), N, True), (dW, second.double(), B, False)):
        a, o = (dz, dz_off) if by_rows else (dz.t().contiguous(), dz_off.t().contiguous())
        want = a @ other
        tol = o @ other.abs() + (n + 8) * U * ((a.abs() + o) @ other.abs()) + unit * want.abs() + (2.0 ** -24 if type == "f16" else 1e-40)
        assert out.dtype == first.dtype and ((out.double() - want).abs() <= tol).all()
    return loss, lse, dH, dW


CODES = [(1, 1, 1, 1, 1, False), (2, 2, 3, 1, 2, False), (63, 1, 200, 3, 5, False), (1000, 3, 256, 5, 512, False), (4097, 4, 64, 2, 10, False), (10_007, 8, 256, 3, 100, False), (10_007, 8, 256, 1, 10, False),
         (5003, 16, 256, 4, 33, False), (3001, 32, 256, 6, 7, False), (1500, 64, 256, 2, 20, False), (700, 128, 256, 1, 300, False), (900, 100, 17, 3, 3, False), (33_333, 8, 256, 130, 50, False),
         (120_001, 8, 256, 2, 100, False), (1_000_003, 4, 256, 1, 10, False), (1, 4, 300, 2, 1, True), (2049, 4, 300, 3, 9, True), (5000, 8, 1024, 5, 100, True), (600, 7, 4096, 2, 64, True), (2000, 1, 16384, 1, 512, True)]


@pytest.mark.parametrize("N,m,b,B,K,wide", CODES)
def test_by_sub_ids(pq, N, m, b, B, K, wide):
    check(pq, *draw_codes(N, m, b, B, K, seed=N + m + B, wide=wide))


DENSE = [(1, 8, 1, 1), (2, 16, 3, 2), (255, 64, 64, 9), (256, 64, 65, 512), (257, 72, 128, 10), (1000, 512, 1, 100), (1003, 512, 50, 33), (5000, 256, 129, 64), (3001, 136, 300, 20), (10_007, 64, 7, 100), (700, 1032, 33, 512),
         (20_003, 8, 64, 300), (9001, 304, 32, 512), (70_001, 512, 64, 100), (40_000, 264, 9, 50), (33_000, 120, 5, 1), (50_001, 512, 100, 30), (70_001, 64, 1030, 7), (12, 512, 64, 512)]


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("N,d,B,K", DENSE)
def test_by_the_default_scorer(pq, N, d, B, K, type):
    check(pq, *draw_dense(N, d, B, K, type, seed=N + d + B), type=type)


@pytest.mark.parametrize("type", list(TYPES))
def test_pieces_of_the_catalogue(pq, type):
    check(pq, *draw_dense(50_003, 32, 4100, 20, type, seed=2), type=type)


@pytest.mark.parametrize("T", [0.5, 2.0, 7.0])
def test_temperatures(pq, T):
    check(pq, *draw_codes(30_001, 8, 256, 5, 30, seed=1), T)
    for type in TYPES:
        check(pq, *draw_dense(30_001, 128, 9, 30, type, seed=2), T, type)
        check(pq, *draw_dense(30_001, 128, 90, 30, type, seed=2), T, type)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("N,d,B", [(3000, 64, 64), (3000, 64, 20), (700, 520, 64), (3000, 64, 70), (1500, 128, 300)])
def test_what_positions_without_a_list_hold_reaches_nothing(pq, N, d, B, type):
    W, H, items, scores, grad = draw_dense(N, d, B, 8, type, seed=N + B)
    items[::3], scores[B - 1] = -1, -np.inf
    clean, odd = H.clone(), H.clone()
    clean[::3], odd[::3] = 0.0, float("nan")
    clean[B - 1], odd[B - 1] = 0.0, float("inf")
    has = torch.ones(B, dtype=torch.bool, device="cuda")
    has[::3], has[B - 1] = False, False
    loss, lse, dH, dW = check(pq, W, clean, items, scores, grad, 1.0, type)
    loss2, lse2 = forward(pq, W, odd, items, scores)
    assert torch.equal(loss, loss2) and torch.equal(lse[has], lse2[has])
    dH2, dW2 = backward(pq, W, odd, items, scores, lse2, grad)
    assert torch.equal(dH, dH2) and torch.equal(dW, dW2) and not dH[~has].any()


@pytest.mark.parametrize("odd", [float("nan"), float("inf")])
@pytest.mark.parametrize("kind", ["u8", "f32", "bf16", "f16", "many"])
def test_lists_that_are_no_numbers_stay_with_their_position(pq, kind, odd):
    type = "bf16" if kind == "many" else kind
    args = draw_codes(3000, 4, 256, 5, 6, seed=3) if kind == "u8" else draw_dense(3000, 64, 90 if kind == "many" else 5, 6, type, seed=3)
    first, second, items, scores, grad = args
    items[2] = torch.tensor([5, 900, 17, 2999, 256, 31], device="cuda")
    bad = scores.clone()
    bad[2, 1] = odd
    clean, got = forward(pq, first, second, items, scores), forward(pq, first, second, items, bad)
    rest = [q for q in range(second.shape[0]) if q != 2]
    assert torch.equal(clean[1], got[1]) and torch.equal(clean[0][rest], got[0][rest]) and got[0][2].isnan()
    out, out_bad = backward(pq, first, second, items, scores, clean[1], grad), backward(pq, first, second, items, bad, clean[1], grad)
    if kind == "u8":
        assert torch.equal(out[rest], out_bad[rest]) and out_bad[2].isnan().all()
        return
    assert torch.equal(out[0][rest], out_bad[0][rest]) and out_bad[0][2].isnan().all()
    others = torch.ones(3000, dtype=torch.bool, device="cuda")
    others[items[2].long()] = False
    assert torch.equal(out[1][others], out_bad[1][others]) and out_bad[1][~others].isnan().all()


@pytest.mark.parametrize("wide", [False, True])
def test_sub_ids_out_of_play(pq, wide):
    codes, S, items, scores, grad = draw_codes(3000, 4, 300 if wide else 256, 5, 8, seed=5, wide=wide)
    S[1, 2] = -np.inf                                           # nothing is left: no loss, no gradient
    S[2, 0, ::2] = -np.inf                                      # listed items among those out of play: the loss is infinite, the gradient is not
    loss, lse, dS = check(pq, codes, S, items, scores, grad)
    assert loss[1] == 0 and not dS[1].any() and loss[2] == np.inf and dS.isfinite().all()


@pytest.mark.parametrize("kind", ["u8", "f32", "many"])
def test_one_entry_is_the_cross_entropy(pq, kind):
    first, second, items, scores, grad = draw_codes(5000, 8, 256, 40, 1, seed=6) if kind == "u8" else draw_dense(5000, 64, 40 if kind == "f32" else 140, 1, "f32", seed=6)
    targets = items[:, 0].contiguous()
    loss, lse = forward(pq, first, second, items, scores)
    if kind == "u8":
        loss2, lse2 = pq.pq_cross_entropy(first, second, targets)
        pairs = [(backward(pq, first, second, items, scores, lse, grad), pq.pq_cross_entropy_backward(first, second, targets, lse2, grad))]
    else:
        loss2, lse2 = pq.pq_default_cross_entropy(first, second, targets)
        pairs = list(zip(backward(pq, first, second, items, scores, lse, grad), pq.pq_default_cross_entropy_backward(first, second, targets, lse2, grad)))
    # the same partial sums (79 of them at most) joined in two orders, 8 and 15 joins deep: a join adds 4 u of a sum (an exponential, a product, an addition,
    # the reference's difference); the logarithm and what it is multiplied with and added to 2 u of the result on either side
    assert ((lse - lse2).abs() <= U * (4 * (8 + 15) + 4 * lse.abs())).all()
    size = scores_of(first, second)[1]
    assert ((loss - loss2).abs() <= U * (4 * size + 66 * size + 64)).all()
    for a, b in pairs:
        assert torch.allclose(a, b, rtol=1e-5, atol=float(140 * U * (size + 64) * b.abs().max()))


def test_gradients_against_differences(pq):
    # central differences of the 64-bit loss: what float32 returns is its derivative to float32's error
    codes, S, items, scores, grad = draw_codes(400, 2, 16, 3, 6, seed=7)
    W, H, items2, scores2, grad2 = draw_dense(300, 8, 3, 6, "f32", seed=8)
    T, h = 2.0, 1e-4

    def objective(first, second, items, scores, grad):
        if first.dtype == torch.uint8:
            z = sum(second[:, k, :][:, first[:, k].long()] for k in range(first.shape[1])) / T
        else:
            z = second @ first.t().contiguous() / T
        w, log_w, any = weights_of(items, scores, first.shape[0], T)
        lp = (z - torch.logsumexp(z, 1, keepdim=True)).gather(1, items.clamp(0, first.shape[0] - 1).long())
        return (grad.double() * T * T * torch.where(w > 0, w * (log_w - lp), 0.0).sum(1)).sum().item()

    _, lse = forward(pq, codes, S, items, scores, T)
    dS = backward(pq, codes, S, items, scores, lse, grad, T)
    _, lse = forward(pq, W, H, items2, scores2, T)
    dH, dW = backward(pq, W, H, items2, scores2, lse, grad2, T)
    for value, gradient, of in ((S.double(), dS, lambda x: objective(codes, x, items, scores, grad)), (H.double(), dH, lambda x: objective(W.double(), x, items2, scores2, grad2)),
                                (W.double(), dW, lambda x: objective(x, H.double(), items2, scores2, grad2))):
        flat = value.view(-1)
        for i in torch.randperm(flat.numel(), generator=torch.Generator().manual_seed(1))[:40].tolist():
            old = flat[i].item()
            flat[i] = old + h
            up = of(value)
            flat[i] = old - h
            down = of(value)
            flat[i] = old
            assert abs((up - down) / (2 * h) - gradient.view(-1)[i].item()) <= 2e-6 * (1 + gradient.abs().max().item())


@pytest.mark.parametrize("kind", ["u8", "bf16", "f16", "many"])
def test_same_bits_every_time_and_on_any_stream(pq, kind):
    args = draw_codes(50_003, 8, 256, 9, 60, seed=9) if kind == "u8" else draw_dense(50_003, 64, 300 if kind == "many" else 9, 60, "f16" if kind == "f16" else "bf16", seed=9)
    first, second, items, scores, grad = args

    def step():
        loss, lse = forward(pq, first, second, items, scores, 2.0)
        out = backward(pq, first, second, items, scores, lse, grad, 2.0)
        return [loss, lse, *([out] if kind == "u8" else out)]

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [step() for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    for got in again:
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("kind", ["u8", "f32", "bf16", "f16", "many"])
def test_in_a_graph(pq, kind):
    type = "bf16" if kind == "many" else kind

    def inputs(seed):
        return draw_codes(20_001, 4, 256, 5, 12, seed) if kind == "u8" else draw_dense(20_001, 64, 130 if kind == "many" else 5, 12, type, seed)

    args = inputs(1)

    def step(first, second, items, scores, grad):
        loss, lse = forward(pq, first, second, items, scores, 2.0)
        out = backward(pq, first, second, items, scores, lse, grad, 2.0)
        return [loss, lse, *([out] if kind == "u8" else out)]

    step(*args)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        outputs = step(*args)
    for seed in (2, 3, 4):
        for to, new in zip(args, inputs(seed)):
            to.copy_(new)
        want = [t.clone() for t in step(*args)]
        for t in outputs:
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outputs))


def test_from_teacher_to_student(pq):
    # the run that these calls are for: a dense teacher's likeliest items are the lists that a head by sub-ids, and a smaller dense one, learn from
    N, B, K, T = 20_011, 96, 40, 2.0
    W, H, _, _, _ = draw_dense(N, 128, B, 1, "bf16", seed=11)
    _, entropy, lse, top, lp = pq.pq_default_log_probs(W, H, None, K, 1.0)
    grad = torch.full((B,), 1.0 / B, device="cuda")
    codes, S, _, _, _ = draw_codes(N, 8, 256, B, 1, seed=12)
    check(pq, codes, S, top, lp, grad, T)
    # lists by ranking scores, whose log-sum nobody asked for, give the same weights: they are a softmax over the list
    ids, ranked = pq.pq_score_topk(codes, S, K)
    _, _, lse8, top8, lp8 = pq.pq_log_probs(codes, S, None, K)
    assert torch.equal(ids, top8)
    w8, w9 = weights_of(top8, lp8, N, T)[0], weights_of(ids, ranked, N, T)[0]
    assert ((w8 - w9).abs() <= w9 * 2 * U * (lp8.abs().max().item() + ranked.abs().max().item()) / T).all()
    W2, H2, _, _, _ = draw_dense(N, 64, B, 1, "f32", seed=13)
    loss, _, dH, dW = check(pq, W2, H2, top8, lp8, grad, T, "f32")
    # a step against the gradient's direction lowers the objective by what the gradient says (to its second order)
    step = 1e-3 / dH.norm().item()
    loss2, _ = pq.pq_default_distillation(W2, H2 - step * dH, top8, lp8, T)
    drop = (loss - loss2).double().mean().item()
    assert abs(drop - step * dH.double().pow(2).sum().item()) <= 0.05 * drop


def test_the_example_runs(pq):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_and_serve.py")
    spec = importlib.util.spec_from_file_location("train_and_serve", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    W, H, _, _, _ = draw_dense(1003, 32, 20, 1, "f32", seed=14)
    losses, alike, log_probs, entropy = example.distillation(W, H, torch.arange(20, dtype=torch.int32, device="cuda"), 32, 4, 256, 3, 5, 2.0, lambda line: None)
    assert len(losses) == 3 and np.isfinite(losses).all() and 0 <= alike <= 1
    assert log_probs.isfinite().all() and (log_probs <= 0).all() and (entropy >= 0).all() and (entropy <= np.log(1003) * (1 + 1e-6)).all()


def test_embeddings_beyond_32_bits_of_offset(pq):
    N, d, B = 4_300_000, 512, 2                                  # 4.4 GB of W and of dW
    W = torch.zeros((N, d), dtype=torch.bfloat16, device="cuda")
    H = torch.ones((B, d), dtype=torch.bfloat16, device="cuda")
    items = torch.tensor([[N - 1, 4_200_001, 17], [4_299_990, -1, -1]], dtype=torch.int32, device="cuda")
    scores = torch.zeros((B, 3), device="cuda")
    loss, lse = forward(pq, W, H, items, scores)
    want = np.log(N) - np.array([np.log(3), 0.0])
    assert np.abs(loss.double().cpu().numpy() - want).max() <= U * (N / 512 + 128)
    _, dW = backward(pq, W, H, items, scores, lse, torch.ones(B, device="cuda"))
    at = torch.tensor([N - 1, 4_200_001, 17, 4_299_990, 5], device="cuda")
    want = torch.tensor([-1 / 3, -1 / 3, -1 / 3, -1.0, 0.0], device="cuda", dtype=torch.float64) + 2 / N
    assert ((dW[at].double() - want[:, None]).abs() <= 2.0 ** -7 * want.abs()[:, None] + 1e-8).all()
    assert ((dW.float().abs() > 1e-3).any(1).sum().item()) == 4
    del W, dW
    torch.cuda.empty_cache()


def test_refusals(pq):
    for first, second, items, scores, grad in (draw_codes(500, 4, 256, 3, 2, seed=1), draw_dense(500, 64, 3, 2, "bf16", seed=1)):
        lse = torch.zeros(3, device="cuda")
        for call, rest in ((forward, ()), (backward, (lse, grad))):
            for T, code in ((0.0, pq.PQ_ERR_SHAPE), (-1.0, pq.PQ_ERR_SHAPE), (float("nan"), pq.PQ_ERR_SHAPE), (1e-5, pq.PQ_ERR_UNSUPPORTED), (float("inf"), pq.PQ_ERR_UNSUPPORTED)):
                with pytest.raises(pq.PQError) as e:
                    call(pq, first, second, items, scores, *rest, T)
                assert e.value.code == code
            with pytest.raises(pq.PQError) as e:
                call(pq, first, second, items[:, :0].contiguous(), scores[:, :0].contiguous(), *rest)
            assert e.value.code in (pq.PQ_ERR_SHAPE, pq.PQ_ERR_NULL)
            with pytest.raises(pq.PQError) as e:
                call(pq, first, second, items.repeat(1, 300), scores.repeat(1, 300), *rest)
            assert e.value.code == pq.PQ_ERR_UNSUPPORTED
            with pytest.raises(pq.PQError) as e:
                call(pq, first, second, items, scores, *rest, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
            assert e.value.code == pq.PQ_ERR_WORKSPACE
            for bad in ((items.long(), scores), (items, scores.double()), (items, scores[:, :1].contiguous()), (items[:2], scores[:2]), (items.cpu(), scores)):
                with pytest.raises(ValueError):
                    call(pq, first, second, *bad, *rest)


@pytest.mark.parametrize("kind", ["u8", "f32", "bf16", "f16", "many"])
def test_one_item_in_every_entry(pq, kind):
    N, K, type = 3_001, 512, "bf16" if kind == "many" else kind
    first, second, items, scores, grad = draw_codes(N, 4, 256, 5, K, seed=21) if kind == "u8" else draw_dense(N, 64, 130 if kind == "many" else 5, K, type, seed=21)
    items[0] = 17                                               # all its entries together have the weight 1
    items[1, ::2] = 0
    items[2] = N - 1
    scores[2] = -np.inf                                         # ... or none
    scores[2, 5] = 1.0
    check(pq, first, second, items, scores, grad, 1.5, None if kind == "u8" else type)


@pytest.mark.parametrize("kind", ["u8", "f32", "bf16", "f16", "many"])
def test_two_steps_at_once(pq, kind):
    type = "bf16" if kind == "many" else kind

    def inputs(seed):
        return draw_codes(60_001, 8, 256, 9, 20, seed) if kind == "u8" else draw_dense(60_001, 64, 200 if kind == "many" else 9, 20, type, seed)

    def step(args):
        loss, lse = forward(pq, *args[:4], 2.0)
        out = backward(pq, *args[:4], lse, args[4], 2.0)
        return [loss, lse, *([out] if kind == "u8" else out)]

    both = [inputs(1), inputs(2)]
    want = [step(each) for each in both]
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, side in enumerate(sides):
            with torch.cuda.stream(side):
                got[i].append(step(both[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for each in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(want[i], each))
