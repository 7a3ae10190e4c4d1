"""The C entry points of the training calls and of the four-bit embeddings on a host without a GPU: they size their workspaces by host
arithmetic and reject bad arguments before any HIP call (so dummy pointers are safe)."""
import ctypes

import pytest

NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGN = -1, -2, -3, -4, -5
P, BIG = 0x10000, 1 << 40
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib(pqlib_path):
    L = ctypes.CDLL(pqlib_path)
    p, i, ll, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t
    for u16 in ("", "_u16"):
        for back in ("", "_backward"):
            f = getattr(L, f"pq_cross_entropy{u16}{back}_workspace_bytes")
            f.argtypes, f.restype = [ll, i, i, i], sz
        getattr(L, f"pq_cross_entropy{u16}").argtypes = [p, p, p, ll, i, i, i, p, p, p, sz, p]
        getattr(L, f"pq_cross_entropy{u16}_backward").argtypes = [p, p, p, p, p, ll, i, i, i, p, p, sz, p]
    L.pq_subitem_scores_backward_workspace_bytes.argtypes, L.pq_subitem_scores_backward_workspace_bytes.restype = [i] * 4, sz
    L.pq_subitem_scores_backward.argtypes = [p] * 5 + [i] * 4 + [p, sz, p]
    for back in ("", "_backward"):
        f = getattr(L, f"pq_default_cross_entropy{back}_workspace_bytes")
        f.argtypes, f.restype = [ll, i, i, i], sz
    L.pq_default_cross_entropy.argtypes = [p, p, p, ll, i, i, i, p, p, p, sz, p]
    L.pq_default_cross_entropy_backward.argtypes = [p] * 5 + [ll, i, i, i, p, p, p, sz, p]
    L.pq_quantise_items.argtypes = [p, ll, i, i, p, p, p]
    L.pq_default_scores_q4.argtypes = [p, p, p, ll, i, i, i, p, ll, p]
    return L


def caller(f, good):
    """Calls f with the named arguments of `good`, some of them replaced."""
    return lambda **other: f(*{**good, **other}.values())


@pytest.mark.parametrize("u16", [False, True])
@pytest.mark.parametrize("backward", [False, True])
def test_cross_entropy_by_sub_ids(lib, u16, backward):
    name = "pq_cross_entropy" + ("_u16" if u16 else "") + ("_backward" if backward else "")
    size = getattr(lib, name + "_workspace_bytes")
    if backward:
        good = dict(codes=P, S=P, targets=P, lse=P, grad=P, N=100_000, B=4, m=8, b=256, dS=P, ws=P, wsb=BIG, stream=None)
        pointers, words = ("codes", "S", "targets", "lse", "grad", "dS", "ws"), ("S", "targets", "lse", "grad", "dS")
    else:
        good = dict(codes=P, S=P, targets=P, N=100_000, B=4, m=8, b=256, loss=P, lse=P, ws=P, wsb=BIG, stream=None)
        pointers, words = ("codes", "S", "targets", "loss", "lse", "ws"), ("S", "targets", "loss", "lse")
    call = caller(getattr(lib, name), good)
    for x in pointers:
        assert call(**{x: None}) == NULL, x
    for x in words:
        assert call(**{x: P + 2}) == ALIGN, x
    assert call(codes=P + 8) == ALIGN and call(ws=P + 8) == ALIGN
    for bad in (dict(N=0), dict(B=0), dict(m=0), dict(b=0), dict(N=2 ** 31), dict(N=-1), dict(b=65537 if u16 else 257)):
        assert call(**bad) == SHAPE, bad
    # 36864 table entries of a query are what LDS holds (one-byte sub-ids of 128 splits always fit)
    for bad in (dict(m=129), dict(B=65536)) + ((dict(m=8, b=4609), dict(m=1, b=36865)) if u16 else (dict(m=145, b=1),)):
        assert call(**bad) == UNSUPPORTED, bad
    shape = lambda **o: tuple({**{k: good[k] for k in ("N", "B", "m", "b")}, **o}.values())
    need = size(*shape())
    assert need > 0 and need % 16 == 0 and call(wsb=need - 1) == WORKSPACE and call(wsb=0) == WORKSPACE
    for bad in (dict(N=0), dict(B=0), dict(m=0), dict(b=0), dict(N=2 ** 31), dict(b=65537), dict(m=129), dict(B=65536)):
        assert size(*shape(**bad)) == 0, bad
    for N, B, m, b in ((1, 1, 1, 1), (10 ** 6, 1, 4, 256), (10 ** 6, 1024, 16, 256), (2 ** 31 - 1, 64, 8, 256), (50_000, 7, 64, 100)):
        need = size(N, B, m, b)
        assert 16 <= need < 2 ** 33 and need % 16 == 0, (N, B, m, b)


def test_python_cuts_no_count_off(pqlib_path):
    from paper_2408_09992_amd import binding as pq
    many = 2 ** 32 + 1                                           # (cut off to an int, one)
    for size in (pq.pq_cross_entropy_workspace_bytes, pq.pq_cross_entropy_backward_workspace_bytes, pq.pq_cross_entropy_u16_workspace_bytes, pq.pq_cross_entropy_u16_backward_workspace_bytes):
        assert size(100, 1, 8, 256) > 0 and size(100, many, 8, 256) == size(100, 1, many, 256) == size(100, 1, 8, many) == 0
    for size in (pq.pq_default_cross_entropy_workspace_bytes, pq.pq_default_cross_entropy_backward_workspace_bytes):
        assert size(100, 1, 64, F32) > 0 and size(100, many, 64, F32) == size(100, 1, 2 ** 32 + 64, F32) == size(100, 1, 64, 2 ** 32) == 0
    size = pq.pq_subitem_scores_backward_workspace_bytes
    assert size(4, 64, 4, 256) > 0 and size(many, 64, 4, 256) == size(4, 64, many, 256) == size(4, 64, 4, many) == 0


def test_largest_tables_by_sub_ids(lib):
    for m, b in ((1, 36864), (2, 18432), (8, 4608), (9, 4096)):
        assert lib.pq_cross_entropy_u16_workspace_bytes(10 ** 5, 3, m, b) > 0 and lib.pq_cross_entropy_u16_backward_workspace_bytes(10 ** 5, 3, m, b) > 0, (m, b)
    assert lib.pq_cross_entropy_workspace_bytes(10 ** 5, 3, 128, 256) > 0 and lib.pq_cross_entropy_backward_workspace_bytes(10 ** 5, 3, 128, 256) > 0


def test_gradients_of_eq4(lib):
    good = dict(dS=P, queries=P, centroids=P, dq=P, dc=P, B=64, d=64, m=4, b=256, ws=P, wsb=BIG, stream=None)
    call = caller(lib.pq_subitem_scores_backward, good)
    assert call(dS=None) == NULL and call(ws=None) == NULL and call(dq=None, dc=None) == NULL
    assert call(centroids=None) == NULL and call(queries=None) == NULL
    for bad in (dict(B=0), dict(d=0), dict(m=0), dict(b=0), dict(d=66), dict(b=65537)):
        assert call(**bad) == SHAPE, bad
    assert call(B=65536) == UNSUPPORTED and call(m=129, d=129) == UNSUPPORTED
    for x in ("dS", "queries", "centroids", "dq", "dc"):
        assert call(**{x: P + 1}) == ALIGN, x
    assert call(ws=P + 4) == ALIGN
    size = lib.pq_subitem_scores_backward_workspace_bytes
    for B in (1, 64, 5000):
        need = size(B, 512, 8, 256)
        assert need >= 16 and need % 16 == 0 and call(B=B, d=512, m=8, wsb=need - 1) == WORKSPACE
    assert size(0, 512, 8, 256) == 0 and size(1, 511, 8, 256) == 0 and size(1, 512, 8, 65537) == 0 and size(65536, 512, 8, 256) == 0


@pytest.mark.parametrize("B", [1, 1000])
def test_gradients_of_eq4_beyond_a_launch(lib, B):
    # 128 splits of 65,536 sub-ids of 1056 elements: more than 2^33 elements of a gradient, 512 threads for every 1024
    good = dict(dS=P, queries=P, centroids=P, dq=P, dc=P, B=B, d=128 * 1056, m=128, b=65536, ws=P, wsb=BIG, stream=None)
    assert caller(lib.pq_subitem_scores_backward, good)() == UNSUPPORTED


@pytest.mark.parametrize("type", [F32, BF16, F16])
@pytest.mark.parametrize("backward", [False, True])
def test_cross_entropy_by_the_default_scorer(lib, type, backward):
    name = "pq_default_cross_entropy" + ("_backward" if backward else "")
    size = getattr(lib, name + "_workspace_bytes")
    if backward:
        good = dict(W=P, queries=P, targets=P, lse=P, grad=P, N=10_000, B=40, d=64, type=type, dq=P, dW=P, ws=P, wsb=BIG, stream=None)
        rows, words = ("W", "queries", "ws", "dq", "dW"), ("targets", "lse", "grad")
    else:
        good = dict(W=P, queries=P, targets=P, N=10_000, B=40, d=64, type=type, loss=P, lse=P, ws=P, wsb=BIG, stream=None)
        rows, words = ("W", "queries", "ws"), ("targets", "loss", "lse")
    call = caller(getattr(lib, name), good)
    for x in rows + words:
        assert call(**{x: None}) == NULL, x
    for x in rows:
        assert call(**{x: P + 8}) == ALIGN, x
    for x in words:
        assert call(**{x: P + 2}) == ALIGN, x
    for bad in (dict(N=0), dict(B=0), dict(d=0), dict(N=2 ** 31), dict(type=3), dict(type=-1)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(B=65536), dict(d=16388), dict(d=66 if type == F32 else 68)):
        assert call(**bad) == UNSUPPORTED, bad
    for N, B, d in ((1, 1, 8), (10_000, 40, 64), (10 ** 6, 1024, 512), (10 ** 6, 64, 512), (2 ** 31 - 1, 300, 512), (1000, 65535, 64)):
        need = size(N, B, d, type)
        assert 16 <= need < 2 ** 33 and need % 16 == 0, (N, B, d)
        assert call(N=N, B=B, d=d, wsb=need - 1) == WORKSPACE
    for bad in ((0, 1, 64, type), (1, 0, 64, type), (1, 1, 0, type), (1, 1, 64, 3), (2 ** 31, 1, 64, type), (1, 65536, 64, type), (1, 1, 2, type)):
        assert size(*bad) == 0, bad


@pytest.mark.parametrize("type", [F32, BF16, F16])
@pytest.mark.parametrize("N,B,d", [(2 ** 27, 65535, 64), (2 ** 31 - 1, 65535, 8), (2 ** 31 - 1, 1000, 512), (2 ** 24, 2048, 128), (10 ** 7, 65535, 64), (2 ** 31 - 1, 1, 8)])
def test_loss_of_long_catalogues_fits_a_launch(lib, type, N, B, d):
    # a sum of 8 bytes a group of items and position; a group has at most 512 threads for 64 positions, and groups come in eights
    groups = lib.pq_default_cross_entropy_workspace_bytes(N, B, d, type) // (8 * B)
    assert groups >= 1 and (groups + 7) // 8 * 8 * ((B + 63) // 64) * 512 < 2 ** 32 and groups * B * 8 < 2 ** 27


def test_four_bit_embeddings(lib):
    make = caller(lib.pq_quantise_items, dict(W=P, N=100, d=128, group=64, packed=P, scales=P, stream=None))
    for x in ("W", "packed", "scales"):
        assert make(**{x: None}) == NULL, x
    score = caller(lib.pq_default_scores_q4, dict(packed=P, scales=P, queries=P, N=100, B=3, d=128, group=64, scores=P, ld=100, stream=None))
    for x in ("packed", "scales", "queries", "scores"):
        assert score(**{x: None}) == NULL, x
    for call in (make, score):
        for bad in (dict(N=0), dict(d=0), dict(N=2 ** 31), dict(group=16), dict(group=0), dict(group=256, d=256), dict(d=96)):
            assert call(**bad) == SHAPE, bad
        assert call(d=16384 + 64) == UNSUPPORTED
        assert call(packed=P + 8) == ALIGN and call(scales=P + 1) == ALIGN
    assert make(W=P + 4) == ALIGN
    assert score(B=0) == SHAPE and score(ld=99) == SHAPE and score(B=65536) == UNSUPPORTED and score(d=9920) == UNSUPPORTED
    assert score(queries=P + 2) == ALIGN and score(scores=P + 1) == ALIGN
