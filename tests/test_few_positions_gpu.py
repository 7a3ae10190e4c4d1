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
