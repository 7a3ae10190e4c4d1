"""The example that trains both heads and serves from them, on a small catalogue."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu


def test_both_heads_learn_their_targets():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_and_serve.py")
    spec = importlib.util.spec_from_file_location("train_and_serve", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.main(items=5003, positions=130, steps=60, d=64, log=lambda line: None)
    # an untrained model knows nothing: about log N; one that has each target well ahead of 5002 others is far below 1
    for losses in (got["sub_ids"], got["default"]):
        assert losses[0] > 0.9 * math.log(5003) and losses[-1] < 0.5
        assert all(math.isfinite(x) for x in losses)
    assert min(got["sub_ids_found"], got["default_found"], got["four_bits_found"]) > 0.95
