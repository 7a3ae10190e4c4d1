"""What the scoring head's distribution over the catalogue costs to ask, and to teach: the operators and their plain forms.

Kinds of case:
  probs-codes    log-probabilities of given items, the entropy and the K likeliest items, by sub-ids (Eq. 5's scores are the logits)
  probs-dense    the same by the default scorer's W phi
  distil-codes   distillation from a teacher's top scores, by sub-ids: loss, log-sum and, in a "step", the gradient with respect to the
                 sub-item score tables
  distil-dense   the same by W phi: in a "step", the gradients of queries and of W

Keys of a case (those a kind needs):
  N d m b   items, embedding width, splits, sub-ids per split;  B  queries (positions)
  n         given items per position (probs);  K  likeliest items asked for (probs), items of a teacher's list (distil)
  T         temperature of the distribution
  pass      "loss": forward only;  "step": forward and backward (distil)
  codes     uniform | zipf: sub-ids drawn uniformly, or by Zipf(1.1) popularity per split
  type      float32 | bfloat16 | float16, of queries and W (dense)
  spread    standard deviation of a position's logits
About one position in twenty has no teacher (padding), and one in ten a shorter list; one given item in twenty is padding.  `own` is set by
whoever measures: false runs the plain forms (elementary torch operations in 32 bits, ranks of dense scores in 64), true the framework's calls.
"""
import math

import torch

own = False

_DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
_PIECE = 1 << 27                     # elements of a piece of logits that the plain forms hold at once


def _probs_codes(N, m, b, B, n, K, T=1.0, codes="uniform", spread=2.5):
    return {"kind": "probs-codes", "N": N, "m": m, "b": b, "B": B, "n": n, "K": K, "T": T, "codes": codes, "spread": spread}


def _probs_dense(N, d, B, n, K, type, T=1.0, spread=2.5):
    return {"kind": "probs-dense", "N": N, "d": d, "B": B, "n": n, "K": K, "T": T, "type": type, "spread": spread}


def _distil_codes(N, m, b, B, K, T, what="step", codes="uniform", spread=2.5):
    return {"kind": "distil-codes", "N": N, "m": m, "b": b, "B": B, "K": K, "T": T, "pass": what, "codes": codes, "spread": spread}


def _distil_dense(N, d, B, K, T, type, what="step", spread=2.5):
    return {"kind": "distil-dense", "N": N, "d": d, "B": B, "K": K, "T": T, "type": type, "pass": what, "spread": spread}


def listed():
    cases = {
        # one user of the smallest catalogue, the probability of what they chose and ten alternatives: latency
        "probs codes tiny 1 position": _probs_codes(10_000, 4, 256, 1, 1, 10),
        # slates of 16 shown items scored for 64 users of a Gowalla-sized catalogue, popular sub-ids
        "probs codes gowalla 64 positions": _probs_codes(1_271_638, 8, 256, 64, 16, 20, 1.0, "zipf"),
        # a teacher's lists of 100 made for a batch, softened
        "probs codes gowalla 512 positions": _probs_codes(1_280_000, 8, 256, 512, 1, 100, 2.0),
        # the dense head of the smallest catalogue, one user: latency
        "probs dense tiny 1 position": _probs_dense(10_000, 64, 1, 1, 10, "float32"),
        # evaluation on a hotel catalogue (Booking.com's 34,742 items), an odd last batch, sampled negatives as given items
        "probs dense booking 203 positions": _probs_dense(34_742, 256, 203, 101, 10, "float16"),
        # serving: 64 users of the large catalogue, bound by W
        "probs dense gowalla 64 positions": _probs_dense(1_271_638, 512, 64, 1, 10, "bfloat16", 0.7),
        # a teacher's lists of 100 made for a training batch, bound by the matrix cores
        "probs dense gowalla 1024 positions": _probs_dense(1_280_000, 512, 1024, 1, 100, "bfloat16", 2.0),
        # a small student by sub-ids, one position: latency
        "distil codes tiny 1 position": _distil_codes(10_000, 4, 256, 1, 10, 1.0),
        # a sub-id head learns from a dense teacher's lists of 100
        "distil codes gowalla 256 positions": _distil_codes(1_271_638, 8, 256, 256, 100, 2.0, "step", "zipf"),
        # 32-bit training on a hotel catalogue
        "distil dense booking 500 positions": _distil_dense(34_742, 512, 500, 50, 2.0, "float32"),
        # few positions of the large catalogue in bfloat16: bound by W and its gradient
        "distil dense gowalla 64 positions": _distil_dense(1_271_638, 512, 64, 100, 1.0, "bfloat16"),
        # a training batch of short embeddings
        "distil dense gowalla 1024 positions": _distil_dense(1_280_000, 256, 1024, 32, 2.0, "bfloat16"),
    }
    return [dict(case, name=name) for name, case in cases.items()]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread evenly over the logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(("probs-codes", "probs-dense", "distil-codes", "distil-dense"))
    T = rng.choice((1.0, 1.0, 0.7, 1.5, 2.0, 4.0))
    spread = round(rng.uniform(1.0, 4.0), 2)
    n = rng.choice((1, 1, 0, _log_int(rng, 2, 128)))
    K = _log_int(rng, 1, 256)
    B = 1 if rng.random() < 0.2 else _log_int(rng, 2, 1024)
    if kind.endswith("codes"):
        m = rng.choices((2, 4, 8, 16, 32), (1, 2, 6, 3, 1))[0]
        b = rng.choice((64, 256, 256, 256, 512, 1024)) if m <= 16 else 256
        N = _log_int(rng, 5_000, max(5_000, min(5_000_000, int(4.0e9 / (B * m)))))
        codes = rng.choice(("uniform", "zipf"))
        if kind == "probs-codes":
            return _probs_codes(N, m, b, B, n, K if rng.random() < 0.9 else 0, T, codes, spread)
        return _distil_codes(N, m, b, B, K, T, rng.choice(("step", "step", "loss")), codes, spread)
    type = rng.choice(("float32", "bfloat16", "bfloat16", "float16"))
    d = rng.choice((64, 128, 200, 256, 512))
    most = 1.0e11 if type == "float32" else 4.0e11
    N = _log_int(rng, 5_000, max(5_000, min(1_280_000, int(most / (B * d)))))
    if kind == "probs-dense":
        return _probs_dense(N, d, B, n, K if rng.random() < 0.9 else 0, type, T, spread)
    return _distil_dense(N, d, B, K, T, type, rng.choice(("step", "step", "loss")), spread)


def _draw_codes(case, gen):
    """Sub-ids int32 [N][m]; a popularity rank per draw, mapped to a sub-id through a permutation per split."""
    N, m, b = case["N"], case["m"], case["b"]
    if case["codes"] == "uniform":
        return torch.randint(0, b, (N, m), dtype=torch.int32, device="cuda", generator=gen)
    weight = torch.arange(1, b + 1, dtype=torch.float64, device="cuda") ** -1.1
    cdf = (weight.cumsum(0) / weight.sum()).float()
    rank = torch.searchsorted(cdf, torch.rand((N, m), device="cuda", generator=gen)).clamp_(max=b - 1)
    order = torch.rand((m, b), device="cuda", generator=gen).argsort(1)
    return torch.stack([order[k][rank[:, k]] for k in range(m)], 1).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(shape, device="cuda", generator=gen)

    s = {"case": case}
    N, B = case["N"], case["B"]

    def ids(*shape):                                             # some items are met more often than others
        return (uniform(*shape).square() * N).to(torch.int32).clamp_(max=N - 1)

    if case["kind"].startswith("probs"):
        items = ids(B, case["n"])
        s["items"] = torch.where(uniform(B, case["n"]) < (0.05 if B * case["n"] > 1 else 0.0), torch.full_like(items, -1), items)
    else:
        K = case["K"]
        listed_items = ids(B, K)
        length = torch.full((B, 1), K, device="cuda")
        kind_of = uniform(B, 1) if B > 1 else torch.ones((B, 1), device="cuda")          # (one position alone has its whole list)
        length = torch.where(kind_of < 0.15, (uniform(B, 1) * K).long() + 1, length)
        length = torch.where(kind_of < 0.05, 0, length)
        s["teacher_items"] = torch.where(torch.arange(K, device="cuda")[None, :] < length, listed_items, torch.full_like(listed_items, -1))
        # a top list: the largest first, falling about as the tail of a normal distribution's does
        s["teacher_scores"] = 12.0 - 1.5 * torch.log1p(torch.arange(K, device="cuda", dtype=torch.float32))[None, :] + 0.1 * normal(B, K)
        s["grad"] = torch.full((B,), 1.0 / B, device="cuda")     # the mean over the batch
    if case["kind"].endswith("codes"):
        codes = _draw_codes(case, gen)
        s["codes"] = codes.to(torch.uint8 if case["b"] <= 256 else torch.uint16)
        s["S"] = normal(B, case["m"], case["b"]) * (case["spread"] * case["m"] ** -0.5)
    else:
        dtype = _DTYPES[case["type"]]
        s["W"] = (normal(N, case["d"]) * case["d"] ** -0.5).to(dtype)
        queries = normal(B, case["d"]) * case["spread"]
        if "teacher_items" in s:                                 # a student that has learnt some of it already
            for k in range(min(4, case["K"])):
                queries += 3.0 * s["W"][s["teacher_items"][:, k].clamp(min=0).long()].float()
        s["queries"] = queries.to(dtype)
    return s


# ---------------------------------------------------------------------------------------------- the framework's calls

def _run_own(s):
    import paper_2408_09992_amd as pq
    case = s["case"]
    T = case["T"]
    wide = case["kind"].endswith("codes") and case["b"] > 256
    if case["kind"].startswith("probs"):
        if case["kind"] == "probs-codes":
            r = (pq.pq_log_probs_u16 if wide else pq.pq_log_probs)(s["codes"], s["S"], s["items"], case["K"], T)
        else:
            r = pq.pq_default_log_probs(s["W"], s["queries"], s["items"], case["K"], T)
        log_probs, entropy, lse, top_items, top_log_probs = r
        return {"log_probs": log_probs, "entropy": entropy, "lse": lse, "top_items": top_items, "top_log_probs": top_log_probs}
    teacher = (s["teacher_items"], s["teacher_scores"])
    if case["kind"] == "distil-codes":
        loss, lse = (pq.pq_distillation_u16 if wide else pq.pq_distillation)(s["codes"], s["S"], *teacher, T)
        if case["pass"] == "loss":
            return {"loss": loss, "lse": lse}
        backward = pq.pq_distillation_u16_backward if wide else pq.pq_distillation_backward
        return {"loss": loss, "lse": lse, "dS": backward(s["codes"], s["S"], *teacher, lse, s["grad"], T)}
    loss, lse = pq.pq_default_distillation(s["W"], s["queries"], *teacher, T)
    if case["pass"] == "loss":
        return {"loss": loss, "lse": lse}
    dqueries, dW = pq.pq_default_distillation_backward(s["W"], s["queries"], *teacher, lse, s["grad"], T)
    return {"loss": loss, "lse": lse, "dqueries": dqueries, "dW": dW}


# ----------------------------------------------------------------------------------------------------- the plain forms

def _pieces(total, rows):
    step = max(1, min(total, _PIECE // max(1, rows)))
    return [(lo, min(total, lo + step)) for lo in range(0, total, step)]


def _scores_by_codes(S, codes):
    index = [codes[:, k].to(torch.int32) for k in range(S.shape[1])]

    def scores(lo, hi):
        z = S[:, 0, :].index_select(1, index[0][lo:hi])
        for k in range(1, len(index)):
            z = z + S[:, k, :].index_select(1, index[k][lo:hi])
        return z + 0.0                                           # (-0 as +0)

    return scores, index


def _scores_of_items(s, items):
    """Scores [B][n] of items [B][n], all of them in the catalogue."""
    if s["case"]["kind"].endswith("codes"):
        S, codes = s["S"], s["codes"].to(torch.int32)
        rows = torch.arange(S.shape[0], device="cuda")[:, None]
        g = codes[items.long()].long()
        z = S[rows, 0, g[:, :, 0]]
        for k in range(1, S.shape[1]):
            z = z + S[rows, k, g[:, :, k]]
        return z + 0.0
    return (s["W"][items.long()].float() * s["queries"].float()[:, None, :]).sum(2)


def _in_order(z):
    """Whole numbers in the order of float32 numbers."""
    bits = z.contiguous().view(torch.int32).to(torch.int64)
    return torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))


def _plain_probs(s):
    case = s["case"]
    N, B, K, T = case["N"], case["B"], case["K"], case["T"]
    by_codes = case["kind"] == "probs-codes"
    if by_codes:
        scores, _ = _scores_by_codes(s["S"], s["codes"])
    else:
        H = s["queries"].float()

        def scores(lo, hi):
            return H @ s["W"][lo:hi].float().t()

    keep = min(N, K + (0 if by_codes else 64))                   # dense: more than K by 32 bits, of which the best K by 64
    top = torch.full((B,), -math.inf, device="cuda")
    total = torch.zeros(B, device="cuda")
    weighted = torch.zeros(B, device="cuda")
    best = torch.empty((B, 0), dtype=torch.int64, device="cuda")
    for lo, hi in _pieces(N, max(B, 1 if by_codes else case["d"])):
        raw = scores(lo, hi)
        z = raw / T
        new_top = torch.maximum(top, z.amax(1))
        shrink = torch.exp(top - new_top)
        top = new_top
        e = torch.exp(z - top[:, None])
        total = total * shrink + e.sum(1)
        weighted = weighted * shrink + (e * z).sum(1)
        if keep:
            key = (_in_order(raw) << 32) + (0x7FFFFFFF - torch.arange(lo, hi, device="cuda"))
            best = torch.cat([best, torch.topk(key, min(keep, hi - lo), dim=1, sorted=False).values], 1)
            best = torch.topk(best, min(keep, best.shape[1]), dim=1).values
    lse = top + torch.log(total)
    entropy = lse - weighted / total
    items = s["items"]
    given = (items >= 0) & (items < N)
    log_probs = torch.where(given, _scores_of_items(s, torch.where(given, items, 0)) / T - lse[:, None], 0.0)
    found = 0x7FFFFFFF - (best & 0xFFFFFFFF)
    if by_codes or not keep:
        found = found[:, :K]
        top_scores = _scores_of_items(s, found)
    else:
        exact_scores = (s["W"][found].double() * s["queries"].double()[:, None, :]).sum(2)
        order = torch.argsort(found, dim=1)                      # by id, then by score without losing that order
        found, exact_scores = found.gather(1, order), exact_scores.gather(1, order)
        order = torch.argsort(exact_scores, dim=1, descending=True, stable=True)[:, :K]
        found, top_scores = found.gather(1, order), exact_scores.gather(1, order).float()
    return {"log_probs": log_probs, "entropy": entropy, "lse": lse, "top_items": found.to(torch.int32), "top_log_probs": top_scores / T - lse[:, None]}


def _plain_distil(s):
    case = s["case"]
    N, B, T = case["N"], case["B"], case["T"]
    by_codes = case["kind"] == "distil-codes"
    items = s["teacher_items"]
    named = (items >= 0) & (items < N)
    u = torch.where(named, s["teacher_scores"] / T, -math.inf)
    highest = u.amax(1, keepdim=True)
    has = highest > -math.inf
    e = torch.where(named, torch.exp(u - torch.where(has, highest, 0.0)), 0.0)
    sums = e.sum(1, keepdim=True)
    weight = torch.where(has, e / torch.where(has, sums, 1.0), 0.0)
    log_weight = u - torch.where(has, highest + torch.log(sums), 0.0)
    if by_codes:
        scores, index = _scores_by_codes(s["S"], s["codes"])
        ids = torch.arange(case["b"], device="cuda", dtype=torch.int32)
    else:
        H = s["queries"].float()

        def scores(lo, hi):
            return H @ s["W"][lo:hi].float().t()

    pieces = _pieces(N, max(B, case["b"] if by_codes else case["d"]))
    top = torch.full((B,), -math.inf, device="cuda")
    total = torch.zeros(B, device="cuda")
    for lo, hi in pieces:
        z = scores(lo, hi) / T
        new_top = torch.maximum(top, z.amax(1))
        total = total * torch.exp(top - new_top) + torch.exp(z - new_top[:, None]).sum(1)
        top = new_top
    lse = top + torch.log(total)
    log_probs = _scores_of_items(s, torch.where(named, items, 0)) / T - lse[:, None]
    loss = T * T * torch.where(weight > 0, weight * (log_weight - log_probs), 0.0).sum(1)
    if case["pass"] == "loss":
        return {"loss": loss, "lse": lse}
    scale = torch.where(has[:, 0], s["grad"] * T, 0.0)
    rows = torch.arange(B, device="cuda")[:, None].expand_as(items)
    if by_codes:
        dS = torch.zeros_like(s["S"])
    else:
        dH, dW = torch.zeros_like(H), torch.empty_like(s["W"])
    for lo, hi in pieces:
        dz = torch.exp(scores(lo, hi) / T - lse[:, None])
        here = named & (items >= lo) & (items < hi)
        dz.index_put_((rows[here], items[here].long() - lo), -weight[here], accumulate=True)
        dz *= scale[:, None]
        if by_codes:
            for k in range(case["m"]):
                dS[:, k, :] += dz @ (index[k][lo:hi, None] == ids).float()
        else:
            dH += dz @ s["W"][lo:hi].float()
            dW[lo:hi] = (dz.t() @ H).to(dW.dtype)
    if by_codes:
        return {"loss": loss, "lse": lse, "dS": dS}
    return {"loss": loss, "lse": lse, "dqueries": dH.to(dW.dtype), "dW": dW}


def run(state):
    if own:
        return _run_own(state)
    return (_plain_probs if state["case"]["kind"].startswith("probs") else _plain_distil)(state)


# ------------------------------------------------------------------------------------------------ definitions, 64 bits

def _logits64(s, case):
    """A function of items lo .. hi - 1: their scores over the temperature [B][hi - lo]."""
    if case["kind"].endswith("codes"):
        S, codes = s["S"].double() / case["T"], s["codes"].to(torch.int64)
        B = case["B"]

        def z_of(lo, hi):
            z = torch.zeros((B, hi - lo), dtype=torch.float64, device="cuda")
            for k in range(case["m"]):
                z += torch.gather(S[:, k, :], 1, codes[lo:hi, k][None, :].expand(B, hi - lo))
            return z
    else:
        H = s["queries"].double() / case["T"]

        def z_of(lo, hi):
            return torch.matmul(s["W"][lo:hi].double(), H.t().contiguous()).t()

    return z_of


def exact(case, seed):
    N, B, K = case["N"], case["B"], case["K"]
    by_codes = case["kind"].endswith("codes")
    if float(N) * B * (case["m"] if by_codes else case["d"] / 8.0) > (1.2e10 if by_codes else 6.0e10):
        return None
    s = prepare(case, seed)
    z_of = _logits64(s, case)
    block = max(1, (1 << 25) // max(B, 1 if by_codes else case["d"]))
    spans = [(lo, min(N, lo + block)) for lo in range(0, N, block)]
    lse = torch.full((B,), -math.inf, dtype=torch.float64, device="cuda")
    for lo, hi in spans:
        lse = torch.logaddexp(lse, torch.logsumexp(z_of(lo, hi), dim=1))
    if case["kind"].startswith("probs"):
        entropy = torch.zeros(B, dtype=torch.float64, device="cuda")
        log_probs = torch.zeros((B, case["n"]), dtype=torch.float64, device="cuda")
        best_z = torch.empty((B, 0), dtype=torch.float64, device="cuda")
        best_i = torch.empty((B, 0), dtype=torch.int64, device="cuda")
        for lo, hi in spans:
            lp = z_of(lo, hi) - lse[:, None]
            entropy -= (lp.exp() * lp).sum(1)
            inside = (s["items"] >= lo) & (s["items"] < hi)
            picked = torch.gather(lp, 1, torch.where(inside, s["items"] - lo, 0).long())
            log_probs = torch.where(inside, picked, log_probs)
            if K:
                v, i = torch.topk(lp, min(K, hi - lo), dim=1)
                best_z, best_i = torch.cat([best_z, v], 1), torch.cat([best_i, i + lo], 1)
                order = torch.argsort(best_z, dim=1, descending=True, stable=True)[:, :K]
                best_z, best_i = best_z.gather(1, order), best_i.gather(1, order)
        # (by sub-ids a rank is that of the float32 sum, Eq. 5's chain: of no 64-bit number)
        return {"log_probs": log_probs, "entropy": entropy, "lse": lse, "top_items": None if by_codes else best_i, "top_log_probs": best_z}
    T = case["T"]
    loss = torch.zeros(B, dtype=torch.float64, device="cuda")
    weights = torch.zeros((B, K), dtype=torch.float64, device="cuda")
    items, u = s["teacher_items"].long(), s["teacher_scores"].double() / T
    for q in range(B):
        at = torch.nonzero((items[q] >= 0) & (items[q] < N)).view(-1)
        if at.numel():
            weights[q, at] = torch.softmax(u[q, at], 0)
    z_at = torch.zeros_like(weights)
    for lo, hi in spans:
        inside = (items >= lo) & (items < hi)
        z_at = torch.where(inside, torch.gather(z_of(lo, hi), 1, torch.where(inside, items - lo, 0)), z_at)
    loss = T * T * (torch.special.xlogy(weights, weights) - weights * (z_at - lse[:, None])).sum(1)
    if case["pass"] == "loss":
        return {"loss": loss, "lse": lse}
    share = s["grad"].double() * T * (weights.sum(1) > 0)
    if by_codes:
        m, b = case["m"], case["b"]
        codes = s["codes"].to(torch.int64)
        mass = torch.zeros((m, B * b), dtype=torch.float64, device="cuda")
        shift = torch.arange(B, device="cuda")[:, None] * b
        for lo, hi in spans:
            p = (z_of(lo, hi) - lse[:, None]).exp().reshape(-1)
            for k in range(m):
                mass[k] += torch.bincount((codes[lo:hi, k][None, :] + shift).view(-1), weights=p, minlength=B * b)
        for k in range(m):
            mass[k] -= torch.bincount((codes[items.clamp(min=0), k] + shift).view(-1), weights=weights.view(-1), minlength=B * b)
        return {"loss": loss, "lse": lse, "dS": mass.view(m, B, b).permute(1, 0, 2) * share[:, None, None]}
    H, W = s["queries"].double(), s["W"]
    dH = torch.zeros_like(H)
    dW = torch.empty((N, case["d"]), dtype=torch.float64, device="cuda")
    row_of = torch.arange(B, device="cuda")[:, None].expand_as(items)
    for lo, hi in spans:
        dz = (z_of(lo, hi) - lse[:, None]).exp().contiguous()
        inside = (items >= lo) & (items < hi)
        dz.index_put_((row_of[inside], items[inside] - lo), -weights[inside], accumulate=True)
        dz *= share[:, None]
        dH += torch.matmul(dz, W[lo:hi].double())
        dW[lo:hi] = torch.matmul(dz.t().contiguous(), H)
    return {"loss": loss, "lse": lse, "dqueries": dH, "dW": dW}


def work(case):
    N, B, K = case["N"], case["B"], case["K"]
    step = case.get("pass") == "step"
    if case["kind"].endswith("codes"):
        m, b = case["m"], case["b"]
        tables = 4.0 * B * m * b
        size = float(N) * m * (1 if b <= 256 else 2)
        if case["kind"] == "probs-codes":
            # m - 1 additions, an exponential, its product with the score and two sums' additions per item
            return {"bytes": size + tables + 8.0 * B * (case["n"] + K + 1), "flops": float(B) * N * (m + 3)}
        # m - 1 additions, an exponential and the sum's addition per item; a step does these again and adds to m places
        return {"bytes": size + tables * (2 if step else 1) + 8.0 * B * (K + 2), "flops": float(B) * N * ((m + 1) * 2 + m if step else m + 1)}
    d = case["d"]
    size = 4 if case["type"] == "float32" else 2
    if case["kind"] == "probs-dense":
        return {"bytes": size * float(d) * (N + B) + 8.0 * B * (case["n"] + K + 1), "flops": 2.0 * B * N * d}
    # the logits, once more in the backward pass (they are not kept), and the two products of their gradient
    return {"bytes": size * float(d) * (N + B) * (2 if step else 1) + 8.0 * B * (K + 2), "flops": (8.0 if step else 2.0) * B * N * d}
