"""Softmax cross entropy of the catalogue by sub-ids, its gradient, and Eq. 4's gradients, against the definitions in 64 bits.

Bounds come from the arithmetic: u = 2^-24 is float32's unit.  A score is a chain of m additions: off by at most m u Z, where
Z is the largest sum of absolute values met.  Its exponential's argument adds some units of the argument, a sum of n terms in
a lane n u of itself, the joins a few units more.  A probability exp(r - lse) carries the errors of r and of lse."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
THREADS = 1024


def draw(N, m, b, B, seed, spread=3.0, wide=False, zipf=False):
    rng = np.random.default_rng(seed)
    p = np.arange(1, b + 1) ** -1.3 if zipf else np.ones(b)
    codes = rng.choice(b, size=(N, m), p=p / p.sum()).astype(np.uint16 if wide else np.uint8)
    S = (rng.standard_normal((B, m, b)) * spread / np.sqrt(m)).astype(np.float32)
    targets = rng.integers(0, N, B).astype(np.int32)
    grad = rng.standard_normal(B).astype(np.float32)
    return codes, S, targets, grad


def reference(codes, S, targets, grad):
    """loss, lse, dS in 64 bits, and the largest sum of absolute values of a score."""
    (N, m), (B, _, b) = codes.shape, S.shape
    loss, lse, dS = np.zeros(B), np.zeros(B), np.zeros((B, m, b))
    mass = np.zeros((B, m, b))
    size = 0.0
    for q in range(B):
        T = S[q].astype(np.float64)
        parts = np.stack([T[k][codes[:, k]] for k in range(m)])
        z = parts.sum(0)
        finite = np.isfinite(z)
        if finite.any():
            size = max(size, np.abs(parts[:, finite]).sum(0).max())
            top = z[finite].max()
            lse[q] = top + np.log(np.exp(z - top).sum())
        else:
            lse[q] = -np.inf
        t = targets[q]
        if not (0 <= t < N) or not np.isfinite(lse[q]):
            continue
        loss[q] = lse[q] - z[t]
        p = np.exp(z - lse[q])
        for k in range(m):
            mass[q, k] = np.bincount(codes[:, k], weights=p, minlength=b)[:b]
            dS[q, k] = mass[q, k]
            dS[q, k, codes[t, k]] -= 1.0
        dS[q] *= float(grad[q])
    return loss, lse, dS, mass, size


def bounds(N, m, size):
    score = U * m * size
    lse = score + U * (N / THREADS + 64 + 4 * size + 4 * np.log(max(N, 2)))
    p = score + lse + U * (4 * size + 64)                      # relative, of a probability
    return score + lse + U * (size + 4), lse, p


def on_gpu(*arrays):
    return [torch.from_numpy(a).cuda() for a in arrays]


def run(pq, codes, S, targets, grad):
    wide = codes.dtype == np.uint16
    c, s, t, g = on_gpu(codes, S, targets, grad)
    forward = pq.pq_cross_entropy_u16 if wide else pq.pq_cross_entropy
    backward = pq.pq_cross_entropy_u16_backward if wide else pq.pq_cross_entropy_backward
    loss, lse = forward(c, s, t)
    dS = backward(c, s, t, lse, g)
    torch.cuda.synchronize()
    return loss.cpu().numpy(), lse.cpu().numpy(), dS.cpu().numpy()


def check(pq, codes, S, targets, grad):
    N, m = codes.shape
    loss, lse, dS = run(pq, codes, S, targets, grad)
    want_loss, want_lse, want_dS, mass, size = reference(codes, S, targets, grad)
    tol_loss, tol_lse, tol_p = bounds(N, m, size)
    same = np.isinf(want_lse)
    assert np.array_equal(lse[same], want_lse[same])
    assert np.all(np.abs(lse[~same] - want_lse[~same]) <= tol_lse)
    same = np.isinf(want_loss)
    assert np.array_equal(loss[same], want_loss[same])
    assert np.all(np.abs(loss[~same] - want_loss[~same]) <= tol_loss)
    g = np.abs(grad.astype(np.float64))[:, None, None]
    assert np.all(np.abs(dS - want_dS) <= g * (mass * tol_p + N * 2.0 ** -62) + 2 * U * np.abs(want_dS) + 1e-44)
    return loss, lse, dS


SHAPES = [(1, 1, 1, 1, False), (2, 2, 3, 1, False), (63, 1, 200, 3, False), (1000, 3, 256, 5, False), (4097, 4, 64, 2, False), (2048, 2, 256, 7, False),
          (10_007, 8, 256, 3, False), (10_007, 8, 256, 1, False), (5003, 16, 256, 4, False), (5003, 16, 256, 1, False), (3001, 32, 256, 6, False),
          (1500, 64, 256, 2, False), (700, 128, 256, 1, False), (900, 100, 17, 3, False), (33_333, 8, 256, 130, False), (120_001, 8, 256, 2, False),
          (1, 4, 300, 2, True), (2049, 4, 300, 3, True), (5000, 8, 1024, 5, True), (1201, 16, 1024, 1, True), (600, 7, 4096, 2, True), (3000, 8, 4096, 2, True),
          (777, 2, 13, 9, True), (2000, 1, 16384, 1, True)]


@pytest.mark.parametrize("N,m,b,B,wide", SHAPES)
def test_loss_and_gradient(pq, N, m, b, B, wide):
    check(pq, *draw(N, m, b, B, seed=N + m + b + B, wide=wide))


@pytest.mark.parametrize("m,B", [(8, 1), (8, 2), (8, 6), (4, 5), (16, 3), (32, 2)])
def test_popular_sub_ids(pq, m, B):
    # most lanes of an instruction add to the same few places
    codes, S, targets, grad = draw(20_011, m, 256, B, seed=m * B, zipf=True)
    codes[: 9000] = 7
    check(pq, codes, S, targets, grad)


@pytest.mark.parametrize("offset,spread", [(0.0, 0.0), (5000.0, 3.0), (-5000.0, 3.0), (0.0, 40.0), (300.0, 200.0)])
def test_scores_far_from_zero(pq, offset, spread):
    codes, S, targets, grad = draw(6007, 8, 256, 5, seed=11, spread=spread)
    check(pq, codes, S + np.float32(offset / 8), targets, grad)


def test_positions_without_a_target(pq):
    codes, S, targets, grad = draw(3000, 8, 256, 9, seed=3)
    targets[[0, 3, 8]] = [-1, 3000, -2147483648]
    loss, lse, dS = check(pq, codes, S, targets, grad)
    assert not loss[[0, 3, 8]].any() and not dS[[0, 3, 8]].any() and np.isfinite(lse).all()
    targets[:] = -1
    loss, lse, dS = check(pq, codes, S, targets, grad)
    assert not loss.any() and not dS.any()


@pytest.mark.parametrize("wide", [False, True])
def test_sub_ids_out_of_play(pq, wide):
    codes, S, targets, grad = draw(5000, 4, 256, 8, seed=5, wide=wide)
    S[0, 1, ::2] = -np.inf                                     # half of a split
    S[1, 2, :] = -np.inf                                       # nothing is left
    S[2, 0, codes[targets[2], 0]] = -np.inf                    # not the target
    only = codes[targets[3]]
    S[3, :, :] = -np.inf
    S[3, np.arange(4), only] = 1.5                             # the target alone
    S[4, 3, 1:] = -np.inf                                      # few items, late in a lane's share
    codes[: 4990, 3] = 1
    codes[4990:, 3] = 0
    loss, lse, dS = check(pq, codes, S, targets, grad)
    assert lse[1] == -np.inf and loss[1] == 0.0 and not dS[1].any()
    assert np.isinf(loss[2]) and np.isfinite(dS[2]).all() and np.isfinite(dS[4]).all()


LOWEST = float(np.finfo(np.float32).min)


@pytest.mark.parametrize("mask", [-1e7, -1e9, -1e10, -1e12, -1e20, -1e30, -1e38, LOWEST])
@pytest.mark.parametrize("m,B,wide", [(8, 1, False), (4, 2, True), (8, 6, False), (3, 5, True), (64, 2, False)])
def test_masks_of_large_finite_numbers(pq, mask, m, B, wide):
    # a score far below any other's counts as -inf, whether a lane meets it before or after the scores that are in play
    codes, S, targets, grad = draw(9000, m, 200, B, seed=m + B, wide=wide)
    codes[:3000, 1] = codes[:3000, 1] // 2
    codes[3000:, 1] = np.where(np.arange(6000) % 3 == 0, codes[3000:, 1] // 2, 100 + codes[3000:, 1] // 2)
    targets[:] = 5000 + 3 * np.arange(B) + 2
    masked, out = S.copy(), S.copy()
    masked[:, 1, :100], out[:, 1, :100] = mask, -np.inf
    if B > 1:
        masked[1, 0, :], out[1, 0, :] = mask, -np.inf            # nothing is left
    got, want = run(pq, codes, masked, targets, grad), check(pq, codes, out, targets, grad)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)
    if B > 1:
        assert got[1][1] == -np.inf and got[0][1] == 0.0 and not got[2][1].any()


@pytest.mark.parametrize("top", [1e7, 1e9, 1e10, 1e12, 1e20, 1e30, -LOWEST])
def test_scores_too_large_for_a_loss(pq, top):
    # float32 scores of that size are whole multiples of a half or more: what they would make of a probability is NaN
    codes, S, targets, grad = draw(5000, 4, 256, 5, seed=12)
    want = run(pq, codes, S, targets, grad)
    S[1, 2, codes[77, 2]] = top
    S[3, 0, :] = top
    loss, lse, dS = run(pq, codes, S, targets, grad)
    rest = [0, 2, 4]
    assert np.isnan(lse[[1, 3]]).all() and np.isnan(loss[[1, 3]]).all() and np.isnan(dS[[1, 3]]).all()
    assert np.array_equal(loss[rest], want[0][rest]) and np.array_equal(lse[rest], want[1][rest]) and np.array_equal(dS[rest], want[2][rest])


@pytest.mark.parametrize("offset", [-4e6, -3e5, 3e5, 4e6])
def test_large_scores_leave_a_gradient(pq, offset):
    # the log-sum is a float32 of that size: probabilities are off by what its rounding is, and no sum of them wraps around
    codes, S, targets, grad = draw(6007, 8, 256, 5, seed=13)
    S = S + np.float32(offset / 8)
    loss, lse, dS = run(pq, codes, S, targets, np.ones_like(grad))
    _, want_lse, _, _, _ = reference(codes, S, targets, np.ones_like(grad))
    unit = float(np.spacing(np.float32(abs(offset))))
    # m roundings of a score's partial sums; the reference's, log-sum's and its product's
    assert np.all(np.abs(lse - want_lse) <= 8 * unit / 2 + 3 * unit)
    for q in range(5):
        sums = dS[q].astype(np.float64)
        sums[np.arange(8), codes[targets[q]]] += 1.0
        sums = sums.sum(1)
        # log-sum, its product with log2 e and the exponent's sum are each rounded by up to a quarter (base 2) at the largest of these
        assert np.all(np.abs(np.log2(sums)) <= 3 * unit * np.log2(np.e)) and np.ptp(sums) <= 1e-5


@pytest.mark.parametrize("m,b,wide", [(8, 256, False), (3, 100, False), (4, 1000, True)])
def test_scores_that_are_no_numbers(pq, m, b, wide):
    # positions 1 and 4 meet a NaN, 3 an infinity; 4 has no target
    codes, S, targets, grad = draw(3000, m, b, 7, seed=m + b, wide=wide)
    targets[4] = -1
    codes_t, S_t, targets_t, grad_t = on_gpu(codes, S, targets, grad)
    loss, lse = (pq.pq_cross_entropy_u16 if wide else pq.pq_cross_entropy)(codes_t, S_t, targets_t)
    dS = (pq.pq_cross_entropy_u16_backward if wide else pq.pq_cross_entropy_backward)(codes_t, S_t, targets_t, lse, grad_t)
    odd = S_t.clone()
    odd[1, 0, int(codes[5, 0])] = odd[4, m - 1, int(codes[7, m - 1])] = float("nan")
    odd[3, 1, int(codes[9, 1])] = float("inf")
    loss2, lse2 = (pq.pq_cross_entropy_u16 if wide else pq.pq_cross_entropy)(codes_t, odd, targets_t)
    dS2 = (pq.pq_cross_entropy_u16_backward if wide else pq.pq_cross_entropy_backward)(codes_t, odd, targets_t, lse2, grad_t)
    rest = [0, 2, 5, 6]
    assert torch.isnan(lse2[[1, 3, 4]]).all() and torch.isnan(loss2[[1, 3]]).all() and torch.isnan(dS2[[1, 3]]).all()
    assert loss2[4] == 0 and not dS2[4].any()
    assert torch.equal(loss2[rest], loss[rest]) and torch.equal(lse2[rest], lse[rest]) and torch.equal(dS2[rest], dS[rest])


def test_gradient_against_differences(pq):
    # along a direction that moves no score by more than 1: the third derivative of log-sum-exp is below 1, so central
    # differences are off by h^2 / 6 and by the losses' own errors over h
    codes, S, targets, grad = draw(4001, 8, 256, 6, seed=21, spread=1.0)
    rng = np.random.default_rng(1)
    D = (rng.uniform(-1, 1, S.shape) / 8).astype(np.float32)
    h = 2.0 ** -6
    up, _, _ = run(pq, codes, S + np.float32(h) * D, targets, grad)
    down, _, _ = run(pq, codes, S - np.float32(h) * D, targets, grad)
    _, _, dS = run(pq, codes, S, targets, np.ones_like(grad))
    size = np.abs(S).max() * 8 + 1
    tol = h * h / 6 + (bounds(4001, 8, size)[0] + 8 * U * size) / h
    slope = (up.astype(np.float64) - down) / (2 * h)
    assert np.all(np.abs(slope - (dS.astype(np.float64) * D).sum((1, 2))) <= tol)


def test_rows_of_the_gradient_sum_to_zero(pq):
    # every split's gradient adds up to g (sum of p - 1) = 0
    codes, S, targets, grad = draw(50_000, 8, 256, 4, seed=8)
    _, _, dS = run(pq, codes, S, targets, grad)
    _, _, tol = bounds(50_000, 8, np.abs(S).max() * 8)
    assert np.all(np.abs(dS.astype(np.float64).sum(2)) <= np.abs(grad)[:, None] * (2 * tol + 512 * U))


@pytest.mark.parametrize("m,b,B,wide", [(8, 256, 1, False), (4, 200, 3, False), (2, 1000, 2, True)])
def test_many_shares(pq, m, b, B, wide):
    # more shares of the items than the threads that join an entry's
    check(pq, *draw(150_001, m, b, B, seed=m + B, wide=wide))


def test_same_bits_every_time_and_on_any_stream(pq):
    codes, S, targets, grad = draw(60_000, 8, 256, 10, seed=9, zipf=True)
    first = run(pq, codes, S, targets, grad)
    second = run(pq, codes, S, targets, grad)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        third = run(pq, codes, S, targets, grad)
    for a, b, c in zip(first, second, third):
        assert np.array_equal(a, b) and np.array_equal(a, c)


def test_in_a_graph(pq):
    codes, S, targets, grad = draw(30_000, 8, 256, 6, seed=10)
    c, s, t, g = on_gpu(codes, S, targets, grad)
    phi, psi = torch.randn(6, 64, device="cuda"), torch.randn(8, 256, 8, device="cuda")
    size = max(pq.pq_cross_entropy_workspace_bytes(30_000, 6, 8, 256), pq.pq_cross_entropy_backward_workspace_bytes(30_000, 6, 8, 256), pq.pq_subitem_scores_backward_workspace_bytes(6, 64, 8, 256))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    loss, lse, dS = torch.empty(6, device="cuda"), torch.empty(6, device="cuda"), torch.empty_like(s)
    dphi, dpsi = torch.empty_like(phi), torch.empty_like(psi)

    def step():
        pq.pq_cross_entropy(c, s, t, ws, loss, lse)
        pq.pq_cross_entropy_backward(c, s, t, lse, g, ws, dS)
        pq.pq_subitem_scores_backward(dS, phi, psi, ws, dphi, dpsi)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        s.add_(0.01 * i)
        step()
        want = [x.clone() for x in (loss, lse, dS, dphi, dpsi)]
        for x in (loss, lse, dS, dphi, dpsi):
            x.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (loss, lse, dS, dphi, dpsi)):
            assert torch.equal(a, b)


def test_codes_beyond_32_bits_of_offset(pq):
    # 4.8 GB of codes: all items have sub-ids 0 but the last, whose score is known
    N, m, b = 600_000_001, 8, 256
    codes = torch.zeros((N, m), dtype=torch.uint8, device="cuda")
    codes[N - 1] = 255
    S = torch.zeros((1, m, b), device="cuda")
    S[:, :, 255] = 20.0 / 8
    targets = torch.tensor([N - 1], dtype=torch.int32, device="cuda")
    loss, lse = pq.pq_cross_entropy(codes, S, targets)
    dS = pq.pq_cross_entropy_backward(codes, S, targets, lse, torch.ones(1, device="cuda"))
    p = np.exp(20.0) / (np.exp(20.0) + N - 1)
    tol = U * (64 + 8 * 20 + N / (256 * THREADS) + 4 * 20.5)
    assert abs(loss.item() + np.log(p)) <= tol and abs(lse.item() - np.log(np.exp(20.0) + N - 1)) <= tol
    assert abs(dS[0, 5, 255].item() - (p - 1)) <= 4 * tol and abs(dS[0, 5, 0].item() - (1 - p)) <= 4 * tol
    assert not dS[0, :, 1:255].any()


@pytest.mark.parametrize("B,d,m,b", [(1, 1, 1, 1), (1, 64, 4, 256), (3, 24, 8, 5), (33, 512, 8, 256), (257, 128, 16, 64), (5, 96, 2, 1000), (64, 96, 3, 33), (1024, 512, 8, 256), (7, 40, 5, 257), (130, 40, 5, 20), (1300, 96, 3, 260), (700, 34, 2, 100), (600, 64, 4, 1000), (2500, 128, 16, 64)])
def test_gradients_of_queries_and_centroids(pq, B, d, m, b):
    rng = np.random.default_rng(B + d + m + b)
    s = d // m
    dS, phi, psi = (rng.standard_normal(shape).astype(np.float32) for shape in ((B, m, b), (B, d), (m, b, s)))
    dphi, dpsi = pq.pq_subitem_scores_backward(*on_gpu(dS, phi, psi))
    x, y, w = dS.astype(np.float64), phi.astype(np.float64).reshape(B, m, s), psi.astype(np.float64)
    # a sum of n products: off by at most n + 8 units of the sum of absolute values
    for got, terms, n in ((dphi.cpu().numpy().reshape(B, m, s), ("qkj,kje->qke", x, w), b), (dpsi.cpu().numpy(), ("qkj,qke->kje", x, y), B)):
        want, size = np.einsum(*terms), np.einsum(terms[0], np.abs(terms[1]), np.abs(terms[2]))
        assert np.all(np.abs(got - want) <= U * (n + 8) * size + 1e-37)


@pytest.mark.parametrize("B", [5, 1300])
def test_one_gradient_alone(pq, B):
    dS, phi, psi = torch.randn(B, 4, 256, device="cuda"), torch.randn(B, 64, device="cuda"), torch.randn(4, 256, 16, device="cuda")
    dphi, dpsi = pq.pq_subitem_scores_backward(dS, phi, psi)
    one, two = torch.zeros_like(phi), torch.zeros_like(psi)
    size = pq.pq_subitem_scores_backward_workspace_bytes(B, 64, 4, 256)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert pq.lib().pq_subitem_scores_backward(dS.data_ptr(), None, psi.data_ptr(), one.data_ptr(), None, B, 64, 4, 256, ws.data_ptr(), size, stream) == 0
    assert pq.lib().pq_subitem_scores_backward(dS.data_ptr(), phi.data_ptr(), None, None, two.data_ptr(), B, 64, 4, 256, ws.data_ptr(), size, stream) == 0
    assert torch.equal(one, dphi) and torch.equal(two, dpsi)


def test_rows_that_are_not_aligned(pq):
    # queries whose rows begin between 16-byte pieces
    B, m, b, s = 1200, 4, 64, 16
    dS, psi = torch.randn(B, m, b, device="cuda"), torch.randn(m, b, s, device="cuda")
    phi = torch.randn(B * m * s + 1, device="cuda")[1:].view(B, m * s)
    for got, want in zip(pq.pq_subitem_scores_backward(dS, phi, psi), pq.pq_subitem_scores_backward(dS, phi.clone(), psi)):
        assert (got - want).abs().max().item() <= 1e-4


def test_refusals_of_the_functions(pq):
    codes, S, targets, grad = on_gpu(*draw(100, 8, 256, 3, seed=1))
    lse = torch.zeros(3, device="cuda")
    with pytest.raises(ValueError):
        pq.pq_cross_entropy(codes.cpu(), S, targets)
    with pytest.raises(ValueError):
        pq.pq_cross_entropy(codes, S.transpose(1, 2), targets)
    with pytest.raises(ValueError):
        pq.pq_cross_entropy(codes, S, targets.long())
    with pytest.raises(ValueError):
        pq.pq_cross_entropy(codes, S, targets[:2])
    with pytest.raises(ValueError):
        pq.pq_cross_entropy_backward(codes, S, targets, lse[:1], grad)
    with pytest.raises(ValueError):
        pq.pq_cross_entropy_backward(codes, S, targets, lse, grad, out=S[:2])
    with pytest.raises(pq.PQError) as e:
        pq.pq_cross_entropy(codes[:, :4].contiguous(), S, targets)
    assert e.value.code == pq.PQ_ERR_SHAPE
    with pytest.raises(pq.PQError) as e:
        pq.pq_cross_entropy_backward(codes, S, targets, lse, grad, workspace=torch.empty(0, dtype=torch.uint8, device="cuda").new_empty(8))
    assert e.value.code == pq.PQ_ERR_WORKSPACE
    with pytest.raises(pq.PQError) as e:
        pq.pq_subitem_scores_backward(S, torch.zeros(3, 30, device="cuda"), torch.zeros(8, 256, 4, device="cuda"))
    assert e.value.code == pq.PQ_ERR_SHAPE


def test_more_positions_than_an_int_counts(pq):
    # 2^32 + 1 of them are not one (the tensors are 17 GB each, of which nothing is read)
    B = 2 ** 32 + 1
    codes = torch.zeros((10, 1), dtype=torch.uint8, device="cuda")
    S, targets = torch.empty((B, 1, 1), device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    with pytest.raises(pq.PQError) as e:
        pq.pq_cross_entropy(codes, S, targets)
    assert e.value.code == pq.PQ_ERR_UNSUPPORTED
    H = S.view(B, 1)
    with pytest.raises(pq.PQError) as e:
        pq.pq_default_cross_entropy(torch.zeros((10, 1), device="cuda"), H, targets)
    assert e.value.code == pq.PQ_ERR_UNSUPPORTED
    with pytest.raises(pq.PQError) as e:
        pq.pq_subitem_scores_backward(S, H, torch.zeros((1, 1, 1), device="cuda"))
    assert e.value.code == pq.PQ_ERR_UNSUPPORTED
