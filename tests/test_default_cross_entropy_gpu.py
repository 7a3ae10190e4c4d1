"""Softmax cross entropy of the catalogue by W phi and its gradients, against the definitions in 64 bits on the same inputs.

u = 2^-24 is float32's unit, U_T the type's (2^-8 bfloat16, 2^-11 float16, u float32).  A score is a float32 sum of d
products: off by at most (d + 2) u times the sum of their absolute values; log-sum and probability as for the sub-ids.  dz is
rounded to the type (relative U_T; float16 besides 2^-40 of the largest |g|), the products sum n terms (n + 8 u of the sum of
absolute values) and are rounded to the type once more."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": (torch.float32, U), "bf16": (torch.bfloat16, 2.0 ** -8), "f16": (torch.float16, 2.0 ** -11)}


def draw(N, d, B, type, seed, spread=2.5):
    rng = np.random.default_rng(seed)
    dtype = TYPES[type][0]
    W = torch.from_numpy((rng.standard_normal((N, d)) * d ** -0.5).astype(np.float32)).to(dtype).cuda()
    H = torch.from_numpy((rng.standard_normal((B, d)) * spread).astype(np.float32)).to(dtype).cuda()
    targets = torch.from_numpy(rng.integers(0, N, B).astype(np.int32)).cuda()
    grad = torch.from_numpy(rng.standard_normal(B).astype(np.float32)).cuda()
    return W, H, targets, grad


def check(pq, W, H, targets, grad, type):
    (N, d), B = W.shape, H.shape[0]
    unit = TYPES[type][1]
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    dH, dW = pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad)
    w, h, g = W.double(), H.double(), grad.double()
    z = (h @ w.t().contiguous())
    size = (h.abs() @ w.abs().t().contiguous()).max().item()
    want_lse = torch.logsumexp(z, 1)
    t = targets.long()
    there = (t >= 0) & (t < N)
    rows = torch.arange(B, device="cuda")
    at = torch.where(there, t, 0)
    want_loss = torch.where(there, want_lse - z[rows, at], torch.zeros_like(want_lse))
    score = (d + 2) * U * size
    tol_lse = score + U * (N / 512 + 64 + 4 * size + 4 * np.log(max(N, 2)))
    assert ((lse.double() - want_lse).abs() <= tol_lse).all()
    assert ((loss.double() - want_loss).abs() <= tol_lse + score + U * (size + 4)).all()
    p = torch.exp(z - want_lse[:, None])
    dz = p.clone()
    dz[rows[there], at[there]] -= 1.0
    g = torch.where(there, g, torch.zeros_like(g))
    dz *= g[:, None]
    rel = score + tol_lse + U * (4 * size + 64)                  # of a probability
    off = g.abs()[:, None] * p * rel + dz.abs() * (unit + 4 * U) + (2.0 ** -40 * g.abs().max() if type == "f16" else 0.0) + 1e-40
    for got, other, n, by_rows in ((dH, w, N, True), (dW, h, B, False)):
        a, o = (dz, off) if by_rows else (dz.t().contiguous(), off.t().contiguous())
        want = a @ other
        tol = o @ other.abs() + (n + 8) * U * ((a.abs() + o) @ other.abs()) + unit * want.abs() + (2.0 ** -24 if type == "f16" else 1e-40)
        assert got.dtype == W.dtype and ((got.double() - want).abs() <= tol).all()
    return loss, lse, dH, dW


SHAPES = [(1, 8, 1), (2, 16, 3), (255, 64, 64), (256, 64, 65), (257, 72, 128), (1000, 512, 1), (1003, 512, 50), (5000, 256, 129), (3001, 136, 300), (10_007, 64, 7), (700, 1032, 33), (4096, 128, 257),
          (70_001, 64, 1030)]


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,d,B", SHAPES)
def test_loss_and_gradients(pq, N, d, B, type):
    check(pq, *draw(N, d, B, type, seed=N + d + B), type)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
def test_pieces_of_the_catalogue(pq, type):
    # more items than a piece holds, an odd number of them
    N, d, B = 50_003, 32, 4100
    assert (N * 4224 > 2 ** 26)
    check(pq, *draw(N, d, B, type, seed=2), type)


@pytest.mark.parametrize("N,d,type", [(70_003, 32, "f32"), (140_003, 72, "bf16")])
def test_pieces_of_longer_rows(pq, N, d, type):
    # more than a gigabyte of dz
    assert N * 4224 * (4 if type == "f32" else 2) > 2 ** 30
    check(pq, *draw(N, d, 4100, type, seed=6), type)


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("N,d,B", [(9001, 304, 40), (20_003, 8, 64), (8200, 328, 1), (5000, 200, 33), (7777, 392, 64), (16_385, 56, 17), (33_000, 120, 5), (3, 512, 64), (70_001, 512, 64), (40_000, 264, 9)])
def test_few_positions(pq, N, d, B, type):
    # several tiles a workgroup, widths that end inside a tile or leave whole parts of it empty
    check(pq, *draw(N, d, B, type, seed=N + d + B), type)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,d,B", [(400_003, 64, 33), (200_100, 128, 40), (50_007, 512, 64), (100_000, 520, 5), (400_000, 56, 100), (200_001, 128, 120), (50_001, 512, 100), (160_007, 64, 300), (80_003, 128, 300),
                                   (9000, 512, 700)])
def test_products_that_fill_the_chip(pq, N, d, B, type):
    # tiles of every height and width, each product in a launch of its own
    check(pq, *draw(N, d, B, type, seed=N + d + B), type)


@pytest.mark.parametrize("d", [4, 12, 20, 36, 100])
def test_float32_widths(pq, d):
    check(pq, *draw(900, d, 70, "f32", seed=d), "f32")


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
def test_positions_without_a_target(pq, type):
    W, H, targets, grad = draw(3000, 64, 70, type, seed=3)
    targets[::3] = -1
    targets[1], targets[69] = 3000, -2147483648
    loss, lse, dH, dW = check(pq, W, H, targets, grad, type)
    assert not loss[::3].any() and not dH[::3].any() and not dH[1].any() and torch.isfinite(lse).all()
    targets[:] = -1
    loss, lse, dH, dW = check(pq, W, H, targets, grad, type)
    assert not loss.any() and not dH.any() and not dW.any()


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,d,B", [(3000, 64, 64), (700, 520, 64), (3000, 64, 70), (1500, 128, 300)])
def test_what_positions_without_a_target_hold_reaches_nothing(pq, N, d, B, type):
    W, H, targets, grad = draw(N, d, B, type, seed=N + B)
    targets[::3], targets[B - 1] = -1, N
    clean, odd = H.clone(), H.clone()
    clean[targets < 0], odd[targets < 0] = 0.0, float("nan")
    clean[B - 1], odd[B - 1] = 0.0, float("inf")
    loss, lse = pq.pq_default_cross_entropy(W, clean, targets)
    loss2, lse2 = pq.pq_default_cross_entropy(W, odd, targets)
    has = (targets >= 0) & (targets < N)
    assert torch.equal(loss, loss2) and torch.equal(lse[has], lse2[has])
    dH, dW = pq.pq_default_cross_entropy_backward(W, clean, targets, lse, grad)
    dH2, dW2 = pq.pq_default_cross_entropy_backward(W, odd, targets, lse2, grad)
    assert torch.equal(dH, dH2) and torch.equal(dW, dW2) and not dH2[~has].any() and torch.isfinite(dW2).all()


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("spread", [0.0, 30.0, 300.0])
def test_scores_far_apart(pq, type, spread):
    check(pq, *draw(2000, 64, 20, type, seed=4, spread=spread), type)


@pytest.mark.parametrize("type,mask", [(t, x) for t in ("f32", "bf16", "f16") for x in (-3e4, -1e10, -1e20, -1e30, -1e38) if t != "f16" or x == -3e4])
@pytest.mark.parametrize("N,d,B", [(5000, 64, 40), (2500, 520, 20), (5000, 64, 300), (70_000, 64, 300)])
def test_items_far_below_any_other(pq, N, d, B, type, mask):
    # an element that is 1 in every query (float16: 30000) takes items out of play, in front of others and between them
    W, H, targets, grad = draw(N, d, B, type, seed=N + d + B)
    H[:, 0], W[:, 0] = (30_000.0 if type == "f16" else 1e4 if mask == -3e4 else 1.0), 0.0
    masked = torch.zeros(N, dtype=torch.bool, device="cuda")
    masked[:N // 3] = True
    masked[N // 2::3] = True
    targets[:] = N // 2 + 1
    targets[1::2] = N // 3 + torch.arange(targets[1::2].numel(), device="cuda", dtype=torch.int32)
    live = torch.nonzero(~masked).view(-1)
    only = W[live].contiguous()
    W[masked, 0] = mask
    among = (torch.cumsum(~masked, 0) - 1)[targets.long()].int()
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    dH, dW = pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad)
    assert not dW[masked].any()
    if type != "f16":                                          # (float16: many targets times 30000 is no float16 any more)
        check(pq, only, H, among, grad, type)
    loss2, lse2 = pq.pq_default_cross_entropy(only, H, among)
    dH2, dW2 = pq.pq_default_cross_entropy_backward(only, H, among, lse2, grad)
    # the same sums in other lanes: some hundred units of a log-sum of about 10, of what makes a gradient besides its type's own
    assert ((lse - lse2).abs() <= 200 * U * 10).all() and ((loss - loss2).abs() <= 200 * U * 20).all()
    unit = TYPES[type][1]
    size = grad.abs()[:, None] * 2 * only[:, 1:].float().abs().max()
    assert ((dH - dH2)[:, 1:].float().abs() <= (6 * unit + 4000 * U) * size).all()
    size = (grad.abs()[:, None] * H[:, 1:].float().abs()).sum(0).max()
    assert ((dW[live] - dW2)[:, 1:].float().abs() <= (6 * unit + 4000 * U) * size).all()


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,d,B", [(3000, 64, 20), (3000, 64, 50), (700, 520, 20), (700, 520, 50), (1500, 128, 300)])
def test_positions_for_which_nothing_is_left(pq, N, d, B, type):
    # as in the loss by sub-ids: log-sum -inf, loss 0, no gradient
    W, H, targets, grad = draw(N, d, B, type, seed=N + B)
    W[:, 0], H[:, 0] = -30_000.0, 0.0
    H[::3, 0], H[::3, 1:] = 60_000.0, 0.0
    targets[1] = -1
    rest = torch.ones(B, dtype=torch.bool, device="cuda")
    rest[::3] = False
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    dH, dW = pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad)
    assert (lse[::3] == -float("inf")).all() and not loss[::3].any() and not dH[::3].any()
    targets[::3] = -1
    loss2, lse2 = pq.pq_default_cross_entropy(W, H, targets)
    dH2, dW2 = pq.pq_default_cross_entropy_backward(W, H, targets, lse2, grad)
    assert torch.isfinite(lse2[rest]).all() and torch.isfinite(dW).all()
    assert torch.equal(loss, loss2) and torch.equal(lse[rest], lse2[rest]) and torch.equal(dH, dH2) and torch.equal(dW, dW2)


def test_gradients_of_very_different_size(pq):
    W, H, targets, grad = draw(2000, 64, 80, "f16", seed=5)
    grad *= torch.logspace(-6, 6, 80, device="cuda")
    grad[7] = 0.0
    W, H = W.float(), H.float()
    check(pq, W, H, targets, grad, "f32")
    check(pq, W.bfloat16(), H.bfloat16(), targets, grad, "bf16")


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("odd", [float("inf"), float("nan")])
@pytest.mark.parametrize("N,d,B", [(3000, 64, 20), (3000, 64, 50), (700, 520, 20), (700, 520, 50), (1500, 128, 300)])
def test_weights_that_are_no_numbers_stay_with_their_position(pq, N, d, B, type, odd):
    W, H, targets, grad = draw(N, d, B, type, seed=N + B)
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    grad[7] = odd
    dH, dW = pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad)
    assert not torch.isfinite(dH[7]).any() and not torch.isfinite(dW[targets[7]]).any()
    grad[7] = 0.0
    dH2, _ = pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad)
    rest = torch.arange(B, device="cuda") != 7
    assert torch.isfinite(dH[rest]).all() and torch.equal(dH[rest], dH2[rest])


def gradients_in_64_bits(W, H, targets, grad):
    """dz, dH, dW and a bound of a probability's relative error (see the head of this file)."""
    (N, d), B = W.shape, H.shape[0]
    w, h = W.double(), H.double()
    z = h @ w.t().contiguous()
    size = (h.abs() @ w.abs().t().contiguous()).max().item()
    dz = torch.exp(z - torch.logsumexp(z, 1)[:, None])
    p = dz.clone()
    dz[torch.arange(B, device="cuda"), targets.long()] -= 1.0
    dz *= grad.double()[:, None]
    score = (d + 2) * U * size
    rel = 2 * score + U * (N / 512 + 128 + 8 * size + 4 * np.log(max(N, 2)))
    return p, dz, dz @ w, dz.t().contiguous() @ h, rel


@pytest.mark.parametrize("N,d,B", [(20_000, 64, 80), (20_000, 64, 40), (20_000, 64, 20), (5000, 512, 64), (3000, 520, 33), (3000, 520, 7), (2000, 128, 300), (100_000, 64, 1030)])
def test_float16_gradients_of_a_position_by_its_own_weight(pq, N, d, B):
    # Weights from 2^12 down to a ten millionth of that.  Every row of dqueries keeps probabilities down to 2^-39 of its own weight (dz is a
    # float16 of p 2^15 and a mantissa of at least a half: half its smallest number is 2^-39 of a probability), dW down to 2^-39 of the largest.
    # For dW queries take their weights' powers of two, below 2^15 and at least 2^14 where that is most: half the smallest is 2^-40 of 2^15, and
    # 2^15 stands for less than four times the largest product of weight and query.
    # (Embeddings of a common mean and scores close together: all probabilities alike, so their roundings do not cancel.)
    W, H, targets, grad = draw(N, d, B, "f16", seed=N + d + B, spread=0.25)
    W += 0.125
    grad = torch.logspace(0, -7, B, device="cuda")[torch.randperm(B, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))] * 4096.0
    grad[::2] *= -1.0
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    dH, dW = pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad)
    p, dz, want_h, want_w, rel = gradients_in_64_bits(W, H, targets, grad)
    unit, g, w, h = TYPES["f16"][1], grad.double().abs()[:, None], W.double().abs(), H.double().abs()
    off = g * p * rel + dz.abs() * (unit + 4 * U)
    tol = (off + 2.0 ** -39 * g) @ w + (N + 8) * U * (dz.abs() @ w) + unit * want_h.abs() + 2.0 ** -24
    assert ((dH.double() - want_h).abs() <= tol).all()
    off = (off + 2.0 ** -39 * g.max()).t().contiguous() @ h
    tol = off + (dz.abs() / g).sum(0)[:, None] * 2.0 ** -38 * (g * h).max() + (B + 8) * U * (dz.abs().t().contiguous() @ h) + unit * want_w.abs() + 2.0 ** -24
    assert ((dW.double() - want_w).abs() <= tol).all()


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 200, 256, 512, 520, 1032])
@pytest.mark.parametrize("N,B", [(50, 1), (700, 1), (60, 2), (1003, 8), (40, 31), (2000, 32), (20_011, 3)])
def test_up_to_32_positions_lose_nothing_to_a_rounded_dz(pq, N, d, B, type):
    # dz is multiplied with what its rounding leaves, so what is left of that rounding is a unit of a unit; then the result's own rounding
    W, H, targets, grad = draw(N, d, B, type, seed=N + d + B, spread=4.0)
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    dH, dW = pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad)
    p, dz, want_h, want_w, rel = gradients_in_64_bits(W, H, targets, grad)
    unit, g, w, h = TYPES[type][1], grad.double().abs()[:, None], W.double().abs(), H.double().abs()
    tiny = 2.0 ** -39 if type == "f16" else 0.0
    floor = 2.0 ** -24 if type == "f16" else 1e-40
    off = g * p * rel + dz.abs() * (unit * unit + 4 * U)
    for got, want, o, a, other, n in ((dH, want_h, off + tiny * g, dz.abs(), w, N),
                                      (dW, want_w, (off + tiny * g.max()).t().contiguous(), dz.abs().t().contiguous(), h, B)):
        tol = o @ other + (n + 8) * U * ((a + o) @ other) + unit * want.abs() * (1 + 2 * unit) + floor
        if type == "f16" and got is dW:
            tol = tol + (dz.abs() / g).sum(0)[:, None] * 2.0 ** -38 * (g * h).max()
        assert ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("weight", [1 / 501, 1 / 110, 1 / 103, 1 / 108, 1.0, 3.0])
@pytest.mark.parametrize("N,d,B", [(5000, 256, 501), (5000, 128, 110), (3000, 512, 50), (3000, 64, 64), (700, 520, 40), (2000, 64, 20)])
def test_one_weight_for_all_adds_no_error_of_its_own(pq, N, d, B, type, weight):
    # The mean square of a gradient's error is that of its own rounding, and of as many independent roundings of dz: below twice the first.
    # (A weight rounded alike in every row of dz would be a common factor.)  A tenth more for what 32 bits do and the draw.
    W, H, targets, grad = draw(N, d, B, type, seed=N + d + B)
    grad.fill_(weight)
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    dH, dW = pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad)
    p, dz, want_h, want_w, rel = gradients_in_64_bits(W, H, targets, grad)
    for got, want in ((dH, want_h), (dW, want_w)):
        own = want.to(W.dtype).double() - want
        assert (got.double() - want).square().sum() <= 1.1 * 2 * own.square().sum()


def test_gradients_against_differences(pq):
    # float32; see the sub-ids' test: directions that move no score by more than 1
    N, d, B = 3000, 64, 9
    W, H, targets, grad = draw(N, d, B, "f32", seed=6, spread=1.0)
    D = torch.randn_like(H)
    D /= (D.double() @ W.double().t().contiguous()).abs().max().float() * 1.01
    E = torch.randn_like(W)
    E /= (H.double() @ E.double().t().contiguous()).abs().max().float() * 1.01
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    dH, dW = pq.pq_default_cross_entropy_backward(W, H, targets, lse, torch.ones_like(grad))
    h = 2.0 ** -6
    size = (H.double().abs() @ W.double().abs().t().contiguous()).max().item() + 1
    noise = (3 * (d + 2) * size + N / 512 + 64 + 8 * size + 4 * np.log(N)) * U / h
    up, down = pq.pq_default_cross_entropy(W, H + h * D, targets)[0], pq.pq_default_cross_entropy(W, H - h * D, targets)[0]
    slope = (up.double() - down.double()) / (2 * h)
    assert ((slope - (dH.double() * D).sum(1)).abs() <= h * h / 6 + 2 * noise).all()
    up, down = pq.pq_default_cross_entropy(W + h * E, H, targets)[0], pq.pq_default_cross_entropy(W - h * E, H, targets)[0]
    slope = ((up.double() - down.double()) / (2 * h)).sum()
    assert abs(slope - (dW.double() * E).sum()) <= B * (h * h / 6 + 2 * noise)


@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_same_bits_every_time_and_on_any_stream(pq, type):
    W, H, targets, grad = draw(20_000, 128, 200, type, seed=7)

    def run():
        loss, lse = pq.pq_default_cross_entropy(W, H, targets)
        return (loss, lse) + pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad)

    first, second = run(), run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        third = run()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_in_a_graph(pq):
    N, d, B = 5000, 64, 90
    W, H, targets, grad = draw(N, d, B, "bf16", seed=8)
    ws = torch.empty(max(pq.pq_default_cross_entropy_workspace_bytes(N, B, d, pq.PQ_BFLOAT16), pq.pq_default_cross_entropy_backward_workspace_bytes(N, B, d, pq.PQ_BFLOAT16)), dtype=torch.uint8, device="cuda")
    loss, lse, dH, dW = torch.empty(B, device="cuda"), torch.empty(B, device="cuda"), torch.empty_like(H), torch.empty_like(W)

    def step():
        pq.pq_default_cross_entropy(W, H, targets, ws, loss, lse)
        pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad, ws, dH, dW)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        H.add_(0.125 * i)
        step()
        want = [x.clone() for x in (loss, lse, dH, dW)]
        for x in (loss, lse, dH, dW):
            x.fill_(7.0)
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (loss, lse, dH, dW)):
            assert torch.equal(a, b)


def test_embeddings_beyond_32_bits_of_offset(pq):
    # 9 GB of W: every item scores 0 but the last one
    N, d = 70_000_001, 64
    W = torch.zeros((N, d), dtype=torch.bfloat16, device="cuda")
    W[N - 1] = 1.0
    H = torch.full((2, d), 0.3125, dtype=torch.bfloat16, device="cuda")
    targets = torch.tensor([N - 1, 3], dtype=torch.int32, device="cuda")
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    want = np.log(np.exp(20.0) + N - 1)
    tol = U * (64 * 20 + N / 512 + 200)
    assert abs(lse[0].item() - want) <= tol and abs(loss[0].item() - (want - 20.0)) <= tol and abs(loss[1].item() - want) <= tol
    dH, dW = pq.pq_default_cross_entropy_backward(W, H, targets, lse, torch.ones(2, device="cuda"))
    p = np.exp(20.0 - want)
    assert abs(dW[N - 1, 5].item() - (2 * p - 1) * 0.3125) <= 2.0 ** -7 and abs(dW[3, 5].item() + 0.3125) <= 2.0 ** -7
    assert abs(dH[0, 0].item() - (p - 1)) <= 2.0 ** -7 and abs(dH[1, 0].item() - p) <= 2.0 ** -7


def test_queries_of_more_than_half_a_billion_elements(pq):
    N, d, B = 40, 8200, 65535
    assert B * d > 2 ** 29
    W, H, targets, grad = draw(N, d, B, "bf16", seed=9, spread=1.0)
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    dH, dW = pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad)
    rows = torch.cat([torch.arange(50), torch.arange(30_000, 30_050), torch.arange(B - 50, B)]).cuda()
    p, dz, want_h, _, rel = gradients_in_64_bits(W, H[rows], targets[rows], grad[rows])
    unit = TYPES["bf16"][1]
    off = grad[rows].double().abs()[:, None] * p * rel + dz.abs() * (unit + 4 * U)
    tol = off @ W.double().abs() + (N + 8) * U * (dz.abs() @ W.double().abs()) + unit * want_h.abs() + 1e-40
    assert ((dH[rows].double() - want_h).abs() <= tol).all() and torch.isfinite(dH).all() and torch.isfinite(dW).all()
    assert (dH.abs().amax(1) > 0).all()


def test_refusals(pq):
    W, H, targets, grad = draw(100, 64, 3, "bf16", seed=1)
    lse = torch.zeros(3, device="cuda")
    with pytest.raises(ValueError):
        pq.pq_default_cross_entropy(W.cpu(), H, targets)
    with pytest.raises(ValueError):
        pq.pq_default_cross_entropy(W, H.float(), targets)
    with pytest.raises(ValueError):
        pq.pq_default_cross_entropy(W.double(), H.double(), targets)
    with pytest.raises(ValueError):
        pq.pq_default_cross_entropy(W, H, targets.long())
    with pytest.raises(ValueError):
        pq.pq_default_cross_entropy(W.t().contiguous().t(), H, targets)
    with pytest.raises(ValueError):
        pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad[:2])
    with pytest.raises(ValueError):
        pq.pq_default_cross_entropy_backward(W, H, targets, lse, grad, dW=W[:50])
    for w, h, code in ((W, H[:, :32].contiguous(), pq.PQ_ERR_SHAPE), (W[:, :12].contiguous(), H[:, :12].contiguous(), pq.PQ_ERR_UNSUPPORTED)):
        with pytest.raises(pq.PQError) as e:
            pq.pq_default_cross_entropy(w, h, targets)
        assert e.value.code == code
    with pytest.raises(pq.PQError) as e:
        pq.pq_default_cross_entropy(W, H, targets, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.code == pq.PQ_ERR_WORKSPACE
