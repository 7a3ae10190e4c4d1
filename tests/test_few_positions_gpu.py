"""The loss by W phi for up to 64 positions of 16 bits on either side of the rule that chooses its kernel, against the definitions in 64 bits."""
import pytest
import torch

import test_default_cross_entropy_gpu as training
import test_distillation_gpu as teaching

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("N,d,B", [(16_384, 512, 33), (16_385, 512, 32), (16_431, 264, 64), (24_607, 504, 1), (311_297, 256, 40), (622_600, 128, 64), (622_593, 72, 3), (1_245_185, 64, 33), (1_245_200, 8, 17)])
def test_loss_and_gradients(pq, N, d, B, type):
    training.check(pq, *training.draw(N, d, B, type, seed=N + d + B), type)


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("N,d,B,K", [(16_399, 512, 40, 20), (311_400, 200, 9, 100)])
def test_distillation(pq, N, d, B, K, type):
    teaching.check(pq, *teaching.draw_dense(N, d, B, K, type, seed=N + d + B), 2.0, type)


@pytest.mark.parametrize("N,d", [(100, 512), (20_001, 512), (320_001, 256)])
def test_positions_behind_the_last_and_elements_behind_a_row(pq, N, d):
    # B positions of a batch are those of a larger one: neither what lies behind the queries nor behind W reaches a result
    W, H, targets, _ = training.draw(N, d, 64, "bf16", seed=N)
    loss, lse = pq.pq_default_cross_entropy(W, H, targets)
    for B in (1, 31, 32, 33, 63):
        room = torch.full((64, d), float("nan"), dtype=H.dtype, device="cuda")
        room[:B] = H[:B]
        some, some_lse = pq.pq_default_cross_entropy(W, room[:B], targets[:B].contiguous())
        assert torch.equal(some, loss[:B]) and torch.equal(some_lse, lse[:B])


@pytest.mark.parametrize("type,d", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("bf16", 512), ("bf16", 40), ("f16", 72), ("f16", 256), ("f16", 504)])
@pytest.mark.parametrize("N,B,K", [(20_000, 64, 100), (20_000, 33, 30), (3_001, 50, 512), (130, 40, 9), (20_000, 20, 100)])
def test_listed_items_gradients_are_rounded_once(pq, type, N, d, B, K):
    # A listed item's dz is held with what its rounding leaves (a unit of the type, squared), so the gradients are off by their own rounding, what float32 leaves, and the rounding of
    # the probabilities of items that are in nobody's list
    W, H, items, scores, grad = teaching.draw_dense(N, d, B, K, type, seed=N + d + B)
    unit, T = teaching.TYPES[type][1], 2.0
    loss, lse = teaching.forward(pq, W, H, items, scores, T)
    dH, dW = teaching.backward(pq, W, H, items, scores, lse, grad, T)
    z, size, off = teaching.scores_of(W, H)
    z, size, off = z / T, size / T, off / T + 2 * teaching.U * size / T
    w, _, any = teaching.weights_of(items, scores, N, T)
    there = (items >= 0) & (items < N)
    at = torch.where(there, items, 0).long()
    p = torch.where(any[:, None], torch.softmax(z, 1), 0.0)
    rows = torch.arange(B, device="cuda")[:, None].expand_as(at)
    dz = p.clone().index_put_((rows, at), torch.where(any[:, None], -w, 0.0), accumulate=True)
    listed = torch.zeros_like(dz).index_put_((rows, at), there.double(), accumulate=True) > 0
    g = torch.where(any, grad.double() * T, 0.0)
    dz *= g[:, None]
    rel = 2 * off + teaching.U * (N / 512 + 128 + 8 * size + 4 * 10)
    of_dz = torch.where(listed, unit ** 2, unit) + 4 * teaching.U
    dz_off = g.abs()[:, None] * p * rel + dz.abs() * of_dz + (2.0 ** -40 * g.abs().max() if type == "f16" else 0.0) + 1e-40
    for out, other, n, by_rows in ((dH, W.double(), N, True), (dW, H.double(), B, False)):
        a, o = (dz, dz_off) if by_rows else (dz.t().contiguous(), dz_off.t().contiguous())
        want = a @ other
        tol = o @ other.abs() + (2 * n + 8) * teaching.U * ((a.abs() + o) @ other.abs()) + unit * want.abs() + (2.0 ** -24 if type == "f16" else 1e-40)
        assert ((out.double() - want).abs() <= tol).all()
