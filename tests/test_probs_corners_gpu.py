"""Corners of the log-probabilities and the distillation: tables that fill LDS."""
import numpy as np
import pytest
import torch

import test_log_probs_gpu as probs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,b,B", [(4, 2544, 3), (8, 1272, 5), (16, 636, 3), (8, 2544, 2), (1, 20352, 3), (8, 1271, 3)])
def test_tables_as_large_as_lds(pq, m, b, B):
    # (Q queries' tables of m b floats and the sums of the waves fill 160 KB to the last 16 bytes)
    probs.check(pq, *probs.draw_codes(20_001, m, b, B, 3, seed=m + b, wide=True), 10)
    probs.check(pq, *probs.draw_codes(3_001, m, b, B, 3, seed=m + b, wide=True), 10)
