"""The C entry points of the log-probabilities and of the distillation on a host without a GPU: they size their workspaces by host arithmetic
and reject bad arguments before any HIP call (so dummy pointers are safe)."""
import ctypes

import pytest

from test_abi_training import ALIGN, BF16, BIG, F16, F32, NULL, P, SHAPE, UNSUPPORTED, WORKSPACE, caller

TEMPERATURES = [(0.0, SHAPE), (-1.0, SHAPE), (float("nan"), SHAPE), (9e-5, UNSUPPORTED), (1.1e4, UNSUPPORTED), (float("inf"), UNSUPPORTED)]


@pytest.fixture(scope="module")
def lib(pqlib_path):
    L = ctypes.CDLL(pqlib_path)
    p, i, ll, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float, ctypes.c_size_t
    for name, pointers, ints, outputs in [("pq_log_probs", 3, 5, 6), ("pq_log_probs_u16", 3, 5, 6), ("pq_default_log_probs", 3, 5, 6), ("pq_distillation", 4, 4, 3), ("pq_distillation_u16", 4, 4, 3),
                                          ("pq_default_distillation", 4, 4, 3), ("pq_distillation_backward", 6, 4, 2), ("pq_distillation_u16_backward", 6, 4, 2),
                                          ("pq_default_distillation_backward", 6, 4, 3)]:
        size = getattr(L, name + "_workspace_bytes")
        size.argtypes, size.restype = [ll, i, i, i, i], sz
        getattr(L, name).argtypes = [p] * pointers + [ll] + [i] * ints + [f] + [p] * outputs + [sz, p]
    return L


def refusals(call, size, good, shape_of, aligned, words, bad_shapes, bad_kinds):
    for x in aligned + words:
        assert call(**{x: None}) == NULL, x
    for x in aligned:
        assert call(**{x: P + 8}) == ALIGN, x
    for x in words:
        assert call(**{x: P + 2}) == ALIGN, x
    for T, code in TEMPERATURES:
        assert call(T=T) == code, T
    for bad in bad_shapes:
        assert call(**bad) == SHAPE and size(*shape_of(**bad)) == 0, bad
    for bad in bad_kinds:
        assert call(**bad) == UNSUPPORTED and size(*shape_of(**bad)) == 0, bad
    need = size(*shape_of())
    assert need >= 16 and need % 16 == 0 and call(wsb=need - 1) == WORKSPACE and call(wsb=0) == WORKSPACE


@pytest.mark.parametrize("u16", [False, True])
def test_log_probs_by_sub_ids(lib, u16):
    name = "pq_log_probs" + ("_u16" if u16 else "")
    good = dict(codes=P, S=P, items=P, N=100_000, B=4, m=8, b=256, n=3, K=10, T=1.0, log_probs=P, entropy=P, lse=P, top_items=P, top_log_probs=P, ws=P, wsb=BIG, stream=None)
    call, size = caller(getattr(lib, name), good), getattr(lib, name + "_workspace_bytes")
    refusals(call, size, good, lambda **o: tuple({**{k: good[k] for k in ("N", "B", "m", "b", "K")}, **o}.values()), ("codes", "ws"),
             ("S", "items", "log_probs", "entropy", "lse", "top_items", "top_log_probs"),
             (dict(N=0), dict(B=0), dict(m=0), dict(b=0), dict(N=2 ** 31), dict(b=65537 if u16 else 257), dict(K=-1), dict(N=9)),
             (dict(m=129), dict(B=65536), dict(K=513)) + ((dict(m=8, b=4609),) if u16 else ()))
    assert call(n=-1) == SHAPE and call(n=65537) == UNSUPPORTED
    # what is not asked for need not be given
    assert call(n=0, items=None, log_probs=None, wsb=0) == WORKSPACE and call(K=0, top_items=None, top_log_probs=None, wsb=0) == WORKSPACE


@pytest.mark.parametrize("type", [F32, BF16, F16])
def test_log_probs_by_the_default_scorer(lib, type):
    good = dict(W=P, queries=P, items=P, N=100_000, B=4, d=64, type=type, n=3, K=10, T=1.0, log_probs=P, entropy=P, lse=P, top_items=P, top_log_probs=P, ws=P, wsb=BIG, stream=None)
    call, size = caller(lib.pq_default_log_probs, good), lib.pq_default_log_probs_workspace_bytes
    refusals(call, size, good, lambda **o: tuple({**{k: good[k] for k in ("N", "B", "d", "type", "K")}, **o}.values()), ("W", "queries", "ws"),
             ("items", "log_probs", "entropy", "lse", "top_items", "top_log_probs"),
             (dict(N=0), dict(B=0), dict(d=0), dict(N=2 ** 31), dict(type=3), dict(type=-1), dict(K=-1), dict(N=9)), (dict(B=65536), dict(d=16388), dict(d=66 if type == F32 else 68), dict(K=513)))
    assert call(n=-1) == SHAPE and call(n=65537) == UNSUPPORTED


@pytest.mark.parametrize("u16", [False, True])
@pytest.mark.parametrize("backward", [False, True])
def test_distillation_by_sub_ids(lib, u16, backward):
    name = "pq_distillation" + ("_u16" if u16 else "") + ("_backward" if backward else "")
    sizes = dict(N=100_000, B=4, m=8, b=256, K=10, T=1.0)
    if backward:
        good = dict(codes=P, S=P, items=P, scores=P, lse=P, grad=P, **sizes, dS=P, ws=P, wsb=BIG, stream=None)
        words = ("S", "items", "scores", "lse", "grad", "dS")
    else:
        good = dict(codes=P, S=P, items=P, scores=P, **sizes, loss=P, lse=P, ws=P, wsb=BIG, stream=None)
        words = ("S", "items", "scores", "loss", "lse")
    refusals(caller(getattr(lib, name), good), getattr(lib, name + "_workspace_bytes"), good,
             lambda **o: tuple({**{k: good[k] for k in ("N", "B", "m", "b", "K")}, **o}.values()), ("codes", "ws"), words,
             (dict(N=0), dict(B=0), dict(m=0), dict(b=0), dict(N=2 ** 31), dict(b=65537 if u16 else 257), dict(K=0)),
             (dict(m=129), dict(B=65536), dict(K=513)) + ((dict(m=8, b=4609),) if u16 else ()))


@pytest.mark.parametrize("type", [F32, BF16, F16])
@pytest.mark.parametrize("backward", [False, True])
def test_distillation_by_the_default_scorer(lib, type, backward):
    name = "pq_default_distillation" + ("_backward" if backward else "")
    sizes = dict(N=100_000, B=40, d=64, type=type, K=10, T=1.0)
    if backward:
        good = dict(W=P, queries=P, items=P, scores=P, lse=P, grad=P, **sizes, dq=P, dW=P, ws=P, wsb=BIG, stream=None)
        aligned, words = ("W", "queries", "dq", "dW", "ws"), ("items", "scores", "lse", "grad")
    else:
        good = dict(W=P, queries=P, items=P, scores=P, **sizes, loss=P, lse=P, ws=P, wsb=BIG, stream=None)
        aligned, words = ("W", "queries", "ws"), ("items", "scores", "loss", "lse")
    refusals(caller(getattr(lib, name), good), getattr(lib, name + "_workspace_bytes"), good,
             lambda **o: tuple({**{k: good[k] for k in ("N", "B", "d", "type", "K")}, **o}.values()), aligned, words,
             (dict(N=0), dict(B=0), dict(d=0), dict(N=2 ** 31), dict(type=3), dict(type=-1), dict(K=0)), (dict(B=65536), dict(d=16388), dict(d=66 if type == F32 else 68), dict(K=513)))


def test_workspaces_of_the_largest_calls(lib):
    # lists take 2 GiB, or room for the first piece and what a cut keeps of every position
    for N, B, K in ((2 ** 31 - 1, 1, 512), (2 ** 31 - 1, 64, 10), (10 ** 7, 1024, 100), (10 ** 6, 65535, 1), (16_384, 7, 512), (1, 1, 1)):
        a, b = lib.pq_log_probs_workspace_bytes(N, B, 8, 256, K), lib.pq_default_log_probs_workspace_bytes(N, B, 64, BF16, K)
        lists = max(2 ** 31, 8 * B * 16384)
        assert 16 <= a <= lists + 2 ** 31 and 16 <= b <= lists + 2 ** 31, (N, B, K, a, b)
        assert lib.pq_log_probs_workspace_bytes(N, B, 8, 256, 0) < 2 ** 31 and lib.pq_default_log_probs_workspace_bytes(N, B, 64, BF16, 0) < 2 ** 31


def test_python_cuts_no_count_off(pqlib_path):
    from paper_2408_09992_amd import binding as pq
    many = 2 ** 32 + 1                                           # (cut off to an int, one)
    for size in (pq.pq_log_probs_workspace_bytes, pq.pq_log_probs_u16_workspace_bytes, pq.pq_distillation_workspace_bytes, pq.pq_distillation_u16_workspace_bytes,
                 pq.pq_distillation_backward_workspace_bytes, pq.pq_distillation_u16_backward_workspace_bytes):
        assert size(100, 1, 8, 256, 5) > 0 and size(100, many, 8, 256, 5) == size(100, 1, many, 256, 5) == size(100, 1, 8, many, 5) == size(100, 1, 8, 256, many) == 0
    for size in (pq.pq_default_log_probs_workspace_bytes, pq.pq_default_distillation_workspace_bytes, pq.pq_default_distillation_backward_workspace_bytes):
        assert size(100, 1, 64, F32, 5) > 0 and size(100, many, 64, F32, 5) == size(100, 1, 2 ** 32 + 64, F32, 5) == size(100, 1, 64, 2 ** 32, 5) == size(100, 1, 64, F32, many) == 0
