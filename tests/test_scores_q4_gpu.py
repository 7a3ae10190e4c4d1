"""Scores from four-bit item embeddings against the definition in 64 bits, and how the embeddings are made.

A score's error: a query element is rounded by at most 2^-31 of a power of two no larger than twice its row's largest, sums
within a group are exact, conversions and the float32 sum over G groups cost G + 8 units of the sum of absolute values."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def draw(N, d, group, B, seed, top=1.0):
    rng = np.random.default_rng(seed)
    packed = rng.integers(0, 256, (N, d // 2), dtype=np.uint8)
    scales = torch.from_numpy(rng.uniform(0.01, 0.02, (N, d // group)).astype(np.float32)).to(torch.bfloat16)
    queries = (rng.standard_normal((B, d)) * top).astype(np.float32)
    return packed, scales, queries


def unpacked(packed, scales):
    N, half = packed.shape
    n = np.empty((N, half * 2))
    n[:, 0::2] = packed & 15
    n[:, 1::2] = packed >> 4
    s = scales.double().numpy()
    return (n - 8) * np.repeat(s, half * 2 // s.shape[1], axis=1)


def check(pq, packed, scales, queries):
    N, G = scales.shape
    got = pq.pq_default_scores_q4(torch.from_numpy(packed).cuda(), scales.cuda(), torch.from_numpy(queries).cuda())
    assert got.shape == (queries.shape[0], (N + 3) // 4 * 4)
    got = got[:, :N].double().cpu().numpy()
    W, phi = unpacked(packed, scales), queries.astype(np.float64)
    size = np.abs(phi) @ np.abs(W).T
    tol = 2.0 ** -30 * np.abs(phi).max(1)[:, None] * np.abs(W).sum(1)[None, :] + U * (G + 8) * size
    assert np.all(np.abs(got - phi @ W.T) <= tol + 1e-44)
    return got


@pytest.mark.parametrize("N,d,group,B", [(1, 32, 32, 1), (1, 64, 64, 1), (3, 128, 128, 2), (16, 96, 32, 5), (17, 64, 32, 4), (33, 160, 32, 3), (1000, 512, 64, 1),
                                         (1003, 512, 128, 16), (4099, 512, 32, 33), (777, 256, 64, 9), (5000, 384, 128, 7), (257, 640, 64, 65), (20_011, 64, 64, 8),
                                         (100, 4096, 128, 40), (50, 9600, 64, 2), (33, 9856, 128, 5), (40, 4800, 32, 3), (15, 1088, 64, 12)])
def test_scores(pq, N, d, group, B):
    check(pq, *draw(N, d, group, B, seed=N + d + group + B))


@pytest.mark.parametrize("top", [1e-42, 1e-30, 1e-3, 1e6, 1e30])
def test_queries_of_any_size(pq, top):
    # (1e-42: a float32 of so small a number has few bits left, and the score's own rounding is a unit of 2^-149)
    packed, scales, queries = draw(200, 256, 64, 3, seed=4, top=top)
    queries[1, :] = 0.0
    queries[2, 3] *= 1000.0
    got = check(pq, packed, scales, queries) if top > 1e-40 else pq.pq_default_scores_q4(torch.from_numpy(packed).cuda(), scales.cuda(), torch.from_numpy(queries).cuda()).cpu().numpy()
    assert not got[1].any() and np.isfinite(got).all()


def test_queries_that_are_no_numbers(pq):
    packed, scales, queries = draw(100, 128, 64, 6, seed=6)
    queries[1, 5], queries[4, 100] = np.inf, np.nan
    got = pq.pq_default_scores_q4(torch.from_numpy(packed).cuda(), scales.cuda(), torch.from_numpy(queries).cuda())[:, :100].cpu().numpy()
    assert np.isnan(got[[1, 4]]).all() and np.isfinite(got[[0, 2, 3, 5]]).all()


def test_extreme_weights(pq):
    packed, scales, queries = draw(64, 512, 128, 4, seed=7)
    packed[:16], packed[16:32] = 0x00, 0xFF
    queries[:] = np.abs(queries)
    queries[1] = 1.0
    check(pq, packed, scales, queries)


def test_row_stride_and_stream(pq):
    packed, scales, queries = draw(999, 256, 64, 3, seed=8)
    p, s, q = torch.from_numpy(packed).cuda(), scales.cuda(), torch.from_numpy(queries).cuda()
    want = pq.pq_default_scores_q4(p, s, q)[:, :999]
    out = torch.full((3, 1024), 5.0, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pq.pq_default_scores_q4(p, s, q, out=out)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :999], want) and (out[:, 999:] == 5.0).all()


def test_packed_beyond_32_bits_of_offset(pq):
    N, d = 70_000_000, 128                                       # 4.5 GB of nibbles
    packed = torch.full((N, d // 2), 0x88, dtype=torch.uint8, device="cuda")
    packed[N - 1] = 0x99
    scales = torch.full((N, 1), 0.5, dtype=torch.bfloat16, device="cuda")
    got = pq.pq_default_scores_q4(packed, scales, torch.ones((1, d), device="cuda"))
    assert got[0, N - 1].item() == 64.0 and not got[0, :N - 1].any()


@pytest.mark.parametrize("N,d,group", [(1, 32, 32), (7, 64, 64), (1001, 512, 64), (333, 384, 128), (20_000, 96, 32)])
def test_quantised_items(pq, N, d, group):
    rng = np.random.default_rng(N)
    W = (rng.standard_normal((N, d)) * d ** -0.5).astype(np.float32)
    W[0, :group] = 0.0
    W[N // 2] *= 1e-20
    packed, scales = pq.pq_quantise_items(torch.from_numpy(W).cuda(), group)
    groups = torch.from_numpy(W).view(N, d // group, group)
    want = (groups.abs().amax(2) / 7.0).to(torch.bfloat16)
    assert torch.equal(scales.cpu(), want)
    s = want.float()[:, :, None]
    n = torch.where(s > 0, torch.round(groups / torch.where(s > 0, s, torch.ones_like(s))).clamp(-8, 7), torch.zeros_like(groups)).view(N, d).to(torch.int32) + 8
    p = packed.cpu().to(torch.int32)
    assert torch.equal(p & 15, n[:, 0::2]) and torch.equal(p >> 4, n[:, 1::2])
    # no weight is further from what stands for it than half a step, and what the rounded scale cuts off at 7 steps
    err = np.abs(unpacked(packed.cpu().numpy(), scales.cpu()) - W).reshape(N, d // group, group)
    assert np.all(err <= (0.5 + 7 * 2.0 ** -8) * want.double().numpy()[:, :, None] + 1e-44)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_groups_that_hold_no_numbers(pq, group):
    W = torch.from_numpy(np.random.default_rng(9).standard_normal((50, 256)).astype(np.float32)).cuda()
    packed, scales = pq.pq_quantise_items(W, group)
    odd = W.clone()
    odd[3, 200], odd[20, 0], odd[49, 255] = float("nan"), float("inf"), -float("inf")
    packed2, scales2 = pq.pq_quantise_items(odd, group)
    hit = torch.zeros(50, 256 // group, dtype=torch.bool, device="cuda")
    hit[3, 200 // group] = hit[20, 0] = hit[49, 255 // group] = True
    assert torch.equal(torch.isnan(scales2), hit) and torch.equal(scales2[~hit], scales[~hit])
    rest = ~hit.repeat_interleave(group // 2, 1)
    assert torch.equal(packed2[rest], packed[rest])
    scores = pq.pq_default_scores_q4(packed2, scales2, W[:2].contiguous())[:, :50]
    assert torch.isnan(scores[:, [3, 20, 49]]).all() and int(torch.isnan(scores).sum()) == 6


def test_ranking_follows_the_scores(pq):
    # quantise, score, rank: the ids are those of the same scores sorted by hand
    W = torch.randn(5000, 128, device="cuda") * 128 ** -0.5
    scores = pq.pq_default_scores_q4(*pq.pq_quantise_items(W, 64), torch.randn(3, 128, device="cuda"))
    ids, best = pq.pq_topk_scores(scores, 20, N=5000)
    order = torch.sort(scores[:, :5000], dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), order.indices[:, :20]) and torch.equal(best, order.values[:, :20])


def test_refusals(pq):
    packed, scales, queries = draw(100, 128, 64, 2, seed=1)
    p, s, q = torch.from_numpy(packed).cuda(), scales.cuda(), torch.from_numpy(queries).cuda()
    with pytest.raises(ValueError):
        pq.pq_default_scores_q4(p.cpu(), s, q)
    with pytest.raises(ValueError):
        pq.pq_default_scores_q4(p, s.float(), q)
    with pytest.raises(ValueError):
        pq.pq_default_scores_q4(p, s, q.t().contiguous().t())
    for bad in ((p, s[:99], q), (p, s, q[:, :64].contiguous()), (p, torch.ones((100, 8), dtype=torch.bfloat16, device="cuda"), q)):
        with pytest.raises(pq.PQError) as e:
            pq.pq_default_scores_q4(*bad)
        assert e.value.code == pq.PQ_ERR_SHAPE
    with pytest.raises(pq.PQError) as e:
        pq.pq_default_scores_q4(p, s, q, out=torch.empty((2, 96), device="cuda"))
    assert e.value.code == pq.PQ_ERR_SHAPE
    with pytest.raises(pq.PQError) as e:
        pq.pq_quantise_items(torch.ones((4, 128), device="cuda"), 16)
    assert e.value.code == pq.PQ_ERR_SHAPE
