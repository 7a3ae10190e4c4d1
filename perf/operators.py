"""What training the scoring head costs, and serving its dense form from four bits: the operators and their plain forms.

Kinds of case:
  codes   the catalogue's softmax cross entropy by sub-ids (Eq. 5's scores are the logits): loss and log-sum of every
          position and, in a "step", the gradient with respect to the sub-item score tables
  dense   the same over the default scorer's W phi: loss, log-sum and, in a "step", the gradients of queries and of W
  eq4     Eq. 4's gradients: what a gradient of the score tables is to queries and sub-item embeddings
  q4      the default scorer's scores from four-bit item embeddings with a scale per group

Keys of a case (those a kind needs):
  N d m b   items, embedding width, splits, sub-ids per split;  B  queries (positions of a training batch)
  pass      "loss": forward only;  "step": forward and backward
  codes     uniform | zipf: sub-ids drawn uniformly, or by Zipf(1.1) popularity per split
  type      float32 | bfloat16 | float16, of queries and W (dense)
  spread    standard deviation of a position's logits
  group     weights that share a scale (q4)
About one position in twenty has no target (padding).  `own` is set by whoever measures: false runs the plain forms
(elementary torch operations in 32 bits), true the framework's calls.
"""
import math

import torch

own = False

_DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
_PIECE = 1 << 28                     # elements of a piece of logits or of one-hot rows that the plain forms hold at once


def _codes_case(N, m, b, B, what, codes="uniform", spread=2.5):
    return {"kind": "codes", "N": N, "m": m, "b": b, "B": B, "pass": what, "codes": codes, "spread": spread}


def _dense_case(N, d, B, type, what="step", spread=2.5):
    return {"kind": "dense", "N": N, "d": d, "B": B, "type": type, "pass": what, "spread": spread}


def _eq4_case(d, m, b, B):
    return {"kind": "eq4", "d": d, "m": m, "b": b, "B": B}


def _q4_case(N, d, group, B):
    return {"kind": "q4", "N": N, "d": d, "group": group, "B": B}


def listed():
    cases = {
        # the smallest catalogue, one position: launches and what the host does around them
        "codes tiny 1 position": _codes_case(10_000, 4, 256, 1, "step"),
        # a Gowalla-sized catalogue, the last positions of 64 users
        "codes gowalla 64 positions": _codes_case(1_280_000, 8, 256, 64, "step"),
        # the data set's own odd number of items, popular sub-ids, a full training batch
        "codes gowalla 1024 positions": _codes_case(1_271_638, 8, 256, 1024, "step", "zipf", 3.5),
        # validation loss over a larger catalogue with finer codes
        "codes finer loss of 16": _codes_case(5_000_000, 16, 256, 16, "loss"),
        # dense head of a small catalogue, an odd batch of short sequences: latency
        "dense tiny 50 positions": _dense_case(10_000, 64, 50, "float32"),
        # dense head of a hotel catalogue (Booking.com's 34,742 items), 32-bit training
        "dense booking 2048 positions": _dense_case(34_742, 512, 2048, "float32"),
        # dense head of the large catalogue in bfloat16: few positions, bound by W
        "dense gowalla 64 positions": _dense_case(1_271_638, 512, 64, "bfloat16"),
        # ... and a training batch, bound by the matrix cores
        "dense gowalla 1024 positions": _dense_case(1_280_000, 512, 1024, "bfloat16"),
        # tables of one query back to its embedding
        "eq4 tiny 1 query": _eq4_case(64, 4, 256, 1),
        # ... of a training batch
        "eq4 1024 queries": _eq4_case(512, 8, 256, 1024),
        # one user of the large catalogue, dense scores from four bits
        "q4 gowalla one user": _q4_case(1_280_000, 512, 64, 1),
        # a batch of users collected over a few milliseconds
        "q4 gowalla 16 users": _q4_case(1_271_638, 512, 128, 16),
    }
    return [dict(case, name=name) for name, case in cases.items()]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread evenly over the logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choices(("codes", "dense", "eq4", "q4"), (4, 4, 1, 2))[0]
    if kind == "codes":
        m = rng.choices((2, 4, 8, 16, 32), (1, 2, 6, 3, 1))[0]
        b = rng.choice((64, 256, 256, 256, 512, 1024)) if m <= 16 else 256
        B = 1 if rng.random() < 0.15 else _log_int(rng, 2, 1024)
        N = _log_int(rng, 5_000, max(5_000, min(5_000_000, int(8.0e9 / (B * m)))))
        return _codes_case(N, m, b, B, rng.choice(("step", "step", "loss")), rng.choice(("uniform", "zipf")), round(rng.uniform(1.0, 4.0), 2))
    if kind == "dense":
        type = rng.choice(("float32", "bfloat16", "bfloat16", "float16"))
        d = rng.choice((64, 128, 256, 512))
        B = _log_int(rng, 1, 2048)
        most = 1.0e11 if type == "float32" else 6.0e11
        N = _log_int(rng, 5_000, max(5_000, min(1_280_000, int(most / (B * d)))))
        return _dense_case(N, d, B, type, rng.choice(("step", "step", "loss")), round(rng.uniform(1.0, 4.0), 2))
    if kind == "eq4":
        m = rng.choice((4, 8, 16))
        return _eq4_case(rng.choice((64, 128, 256, 512)), m, rng.choice((64, 256, 256, 1024)), _log_int(rng, 1, 2048))
    B = rng.choice((1, 1, 1, 2, 3, 4, 8, 13, 16, 32))
    d = rng.choice((64, 128, 256, 512))
    group = rng.choice([g for g in (32, 64, 128) if g <= d])
    return _q4_case(_log_int(rng, 5_000, 5_000_000 if B <= 4 else 1_280_000), d, group, B)


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

    s = {"case": case}
    B = case["B"]
    if case["kind"] in ("codes", "dense"):
        targets = torch.randint(0, case["N"], (B,), dtype=torch.int32, device="cuda", generator=gen)
        padded = torch.rand(B, device="cuda", generator=gen) < 0.05
        s["targets"] = torch.where(padded, torch.full_like(targets, -1), targets)
        s["grad"] = torch.full((B,), 1.0 / B, device="cuda")           # the mean over the batch
    if case["kind"] == "codes":
        codes = _draw_codes(case, gen)
        s["codes"] = codes.to(torch.uint8 if case["b"] <= 256 else torch.uint16)
        s["S"] = normal(B, case["m"], case["b"]) * (case["spread"] * case["m"] ** -0.5)
    elif case["kind"] == "dense":
        dtype = _DTYPES[case["type"]]
        s["W"] = (normal(case["N"], case["d"]) * case["d"] ** -0.5).to(dtype)
        s["queries"] = (normal(B, case["d"]) * case["spread"]).to(dtype)
    elif case["kind"] == "eq4":
        m, b, d = case["m"], case["b"], case["d"]
        # gradients of score tables: a share of the mean for every sub-id, less the target's
        s["dS"] = torch.rand((B, m, b), device="cuda", generator=gen) * (2.0 / (B * b))
        hit = torch.randint(0, b, (B, m, 1), device="cuda", generator=gen)
        s["dS"].scatter_add_(2, hit, torch.full((B, m, 1), -1.0 / B, device="cuda"))
        s["queries"] = normal(B, d)
        s["centroids"] = normal(m, b, d // m) * d ** -0.5
    else:
        N, d = case["N"], case["d"]
        s["packed"] = torch.randint(0, 256, (N, d // 2), dtype=torch.uint8, device="cuda", generator=gen)
        s["scales"] = ((1.0 + torch.rand((N, d // case["group"]), device="cuda", generator=gen)) * (0.2 * d ** -0.5)).to(torch.bfloat16)
        s["queries"] = normal(B, d)
    return s


# ---------------------------------------------------------------------------------------------- the framework's calls

def _run_own(s):
    import paper_2408_09992_amd as pq
    case = s["case"]
    if case["kind"] == "codes":
        wide = case["b"] > 256
        loss, lse = (pq.pq_cross_entropy_u16 if wide else pq.pq_cross_entropy)(s["codes"], s["S"], s["targets"])
        if case["pass"] == "loss":
            return {"loss": loss, "lse": lse}
        backward = pq.pq_cross_entropy_u16_backward if wide else pq.pq_cross_entropy_backward
        return {"loss": loss, "lse": lse, "dS": backward(s["codes"], s["S"], s["targets"], lse, s["grad"])}
    if case["kind"] == "dense":
        loss, lse = pq.pq_default_cross_entropy(s["W"], s["queries"], s["targets"])
        if case["pass"] == "loss":
            return {"loss": loss, "lse": lse}
        dqueries, dW = pq.pq_default_cross_entropy_backward(s["W"], s["queries"], s["targets"], lse, s["grad"])
        return {"loss": loss, "lse": lse, "dqueries": dqueries, "dW": dW}
    if case["kind"] == "eq4":
        dqueries, dcentroids = pq.pq_subitem_scores_backward(s["dS"], s["queries"], s["centroids"])
        return {"dqueries": dqueries, "dcentroids": dcentroids}
    return {"scores": pq.pq_default_scores_q4(s["packed"], s["scales"], s["queries"])[:, :case["N"]]}


# ----------------------------------------------------------------------------------------------------- the plain forms

def _pieces(total, rows):
    step = max(1, min(total, _PIECE // max(1, rows)))
    return [(lo, min(total, lo + step)) for lo in range(0, total, step)]


def _plain_cross_entropy(logits, pieces, targets, grad, gradients):
    """Loss and log-sum from pieces of logits; gradients(lo, hi, dlogits) for each piece if a gradient is asked for."""
    B = targets.shape[0]
    top = torch.full((B,), -math.inf, device="cuda")
    total = torch.zeros(B, device="cuda")
    picked = torch.zeros(B, device="cuda")
    has_target = targets >= 0
    rows = torch.arange(B, device="cuda")

    def within(lo, hi):
        inside = (targets >= lo) & (targets < hi)
        return inside, torch.where(inside, targets - lo, 0).long()

    for lo, hi in pieces:
        z = logits(lo, hi)
        new_top = torch.maximum(top, z.amax(1))
        total = total * torch.exp(top - new_top) + torch.exp(z - new_top[:, None]).sum(1)
        top = new_top
        inside, at = within(lo, hi)
        picked = torch.where(inside, z[rows, at], picked)
    lse = top + torch.log(total)
    loss = torch.where(has_target, lse - picked, 0.0)
    if gradients is not None:
        scale = torch.where(has_target, grad, 0.0)
        for lo, hi in pieces:
            p = torch.exp(logits(lo, hi) - lse[:, None])
            inside, at = within(lo, hi)
            p[rows, at] -= inside.float()
            gradients(lo, hi, p * scale[:, None])
    return loss, lse


def _plain_codes(s):
    case, S, codes = s["case"], s["S"], s["codes"]
    B, m, b = S.shape
    index = [codes[:, k].to(torch.int32) for k in range(m)]

    def logits(lo, hi):
        z = S[:, 0, :].index_select(1, index[0][lo:hi])
        for k in range(1, m):
            z = z + S[:, k, :].index_select(1, index[k][lo:hi])
        return z

    dS = torch.zeros_like(S)
    ids = torch.arange(b, device="cuda", dtype=torch.int32)

    def gradients(lo, hi, dz):
        for k in range(m):
            dS[:, k, :] += dz @ (index[k][lo:hi, None] == ids).float()

    step = case["pass"] == "step"
    loss, lse = _plain_cross_entropy(logits, _pieces(case["N"], max(B, b)), s["targets"], s["grad"], gradients if step else None)
    return {"loss": loss, "lse": lse, "dS": dS} if step else {"loss": loss, "lse": lse}


def _plain_dense(s):
    case, W = s["case"], s["W"]
    H = s["queries"].float()

    def logits(lo, hi):
        return H @ W[lo:hi].float().t()

    dH = torch.zeros_like(H)
    dW = torch.empty_like(W)

    def gradients(lo, hi, dz):
        dH.add_(dz @ W[lo:hi].float())
        dW[lo:hi] = (dz.t() @ H).to(W.dtype)

    step = case["pass"] == "step"
    loss, lse = _plain_cross_entropy(logits, _pieces(case["N"], max(case["B"], case["d"])), s["targets"], s["grad"], gradients if step else None)
    return {"loss": loss, "lse": lse, "dqueries": dH.to(W.dtype), "dW": dW} if step else {"loss": loss, "lse": lse}


def _plain_eq4(s):
    dS, queries, centroids = s["dS"], s["queries"], s["centroids"]
    m, b, width = centroids.shape
    dqueries = torch.cat([dS[:, k, :] @ centroids[k] for k in range(m)], 1)
    dcentroids = torch.stack([dS[:, k, :].t() @ queries[:, k * width:(k + 1) * width] for k in range(m)])
    return {"dqueries": dqueries, "dcentroids": dcentroids}


def _plain_q4(s):
    case, packed, scales, queries = s["case"], s["packed"], s["scales"], s["queries"]
    N, d = case["N"], case["d"]
    scores = torch.empty((case["B"], N), device="cuda")
    for lo, hi in _pieces(N, d):
        p = packed[lo:hi]
        n = torch.stack((p & 15, p >> 4), 2).view(hi - lo, d // case["group"], case["group"]).float() - 8.0
        W = (n * scales[lo:hi].float()[:, :, None]).view(hi - lo, d)
        scores[:, lo:hi] = queries @ W.t()
    return {"scores": scores}


_PLAIN = {"codes": _plain_codes, "dense": _plain_dense, "eq4": _plain_eq4, "q4": _plain_q4}


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------ definitions, 64 bits

def _exact_rows(z_of, N, B, targets, step_items):
    """log-sum and loss in 64 bits, one block of items after the other."""
    lse = torch.full((B,), -math.inf, dtype=torch.float64, device="cuda")
    for lo in range(0, N, step_items):
        lse = torch.logaddexp(lse, torch.logsumexp(z_of(lo, min(N, lo + step_items)), dim=1))
    loss = torch.zeros(B, dtype=torch.float64, device="cuda")
    return lse, loss


def exact(case, seed):
    s = prepare(case, seed)
    B = case["B"]
    if case["kind"] == "codes":
        N, m, b = case["N"], case["m"], case["b"]
        if float(N) * B * m > 2.5e10:
            return None
        S = s["S"].double()
        codes = s["codes"].to(torch.int64)
        block = max(1, (1 << 26) // B)

        def z_of(lo, hi):
            z = torch.zeros((B, hi - lo), dtype=torch.float64, device="cuda")
            for k in range(m):
                z += torch.gather(S[:, k, :], 1, codes[lo:hi, k][None, :].expand(B, hi - lo))
            return z

        lse, loss = _exact_rows(z_of, N, B, s["targets"], block)
        for q, t in enumerate(s["targets"].tolist()):
            if t >= 0:
                loss[q] = lse[q] - S[q, torch.arange(m, device="cuda"), codes[t]].sum()
        if case["pass"] == "loss":
            return {"loss": loss, "lse": lse}
        mass = torch.zeros((m, B * b), dtype=torch.float64, device="cuda")
        shift = torch.arange(B, device="cuda")[:, None] * b
        for lo in range(0, N, block):
            hi = min(N, lo + block)
            p = (z_of(lo, hi) - lse[:, None]).exp().view(-1)
            for k in range(m):
                mass[k] += torch.bincount((codes[lo:hi, k][None, :] + shift).view(-1), weights=p, minlength=B * b)
        dS = mass.view(m, B, b).permute(1, 0, 2).contiguous()
        for q, t in enumerate(s["targets"].tolist()):
            if t >= 0:
                dS[q, torch.arange(m, device="cuda"), codes[t]] -= 1.0
                dS[q] *= float(s["grad"][q])
            else:
                dS[q] = 0.0
        return {"loss": loss, "lse": lse, "dS": dS}
    if case["kind"] == "dense":
        N, d = case["N"], case["d"]
        H = s["queries"].double()
        block = max(1, (1 << 26) // max(B, d))

        def z_of(lo, hi):
            return torch.matmul(s["W"][lo:hi].double(), H.t()).t()

        lse, loss = _exact_rows(z_of, N, B, s["targets"], block)
        t = s["targets"].long()
        there = t >= 0
        loss[there] = lse[there] - (H[there] * s["W"][t[there]].double()).sum(1)
        if case["pass"] == "loss":
            return {"loss": loss, "lse": lse}
        scale = s["grad"].double() * there
        dH = torch.zeros_like(H)
        dW = torch.empty((N, d), dtype=torch.float64, device="cuda")
        for lo in range(0, N, block):
            hi = min(N, lo + block)
            dz = (z_of(lo, hi) - lse[:, None]).exp()
            mine = torch.nonzero((t >= lo) & (t < hi)).view(-1)
            dz.index_put_((mine, t[mine] - lo), torch.full((mine.numel(),), -1.0, dtype=torch.float64, device="cuda"), accumulate=True)
            dz *= scale[:, None]
            dH += torch.matmul(dz, s["W"][lo:hi].double())
            dW[lo:hi] = torch.matmul(dz.t().contiguous(), H)
        return {"loss": loss, "lse": lse, "dqueries": dH, "dW": dW}
    if case["kind"] == "eq4":
        dS, phi, psi = s["dS"].double(), s["queries"].double(), s["centroids"].double()
        m, b, width = psi.shape
        dphi = torch.empty_like(phi)
        dpsi = torch.empty_like(psi)
        for k in range(m):
            part = slice(k * width, (k + 1) * width)
            dphi[:, part] = torch.matmul(dS[:, k].contiguous(), psi[k])
            dpsi[k] = torch.matmul(dS[:, k].t().contiguous(), phi[:, part].contiguous())
        return {"dqueries": dphi, "dcentroids": dpsi}
    N, d, group = case["N"], case["d"], case["group"]
    phi = s["queries"].double()
    scores = torch.empty((B, N), dtype=torch.float64, device="cuda")
    block = max(1, (1 << 26) // d)
    for lo in range(0, N, block):
        byte = s["packed"][lo:lo + block].to(torch.int64)
        value = torch.empty((byte.shape[0], d), dtype=torch.float64, device="cuda")
        value[:, 0::2] = (byte % 16 - 8).double()
        value[:, 1::2] = (byte // 16 - 8).double()
        value *= s["scales"][lo:lo + block].double().repeat_interleave(group, dim=1)
        scores[:, lo:lo + block] = torch.matmul(value, phi.t()).t()
    return {"scores": scores}


def work(case):
    B = case["B"]
    if case["kind"] == "codes":
        N, m, b = case["N"], case["m"], case["b"]
        step = case["pass"] == "step"
        tables = 4.0 * B * m * b
        # m - 1 additions, an exponential and the sum's addition per item; a step does these again and adds to m places
        return {"bytes": float(N) * m * (1 if b <= 256 else 2) + tables * (2 if step else 1) + 16.0 * B,
                "flops": float(B) * N * ((m + 1) * 2 + m if step else m + 1)}
    if case["kind"] == "dense":
        N, d = case["N"], case["d"]
        step = case["pass"] == "step"
        size = 4 if case["type"] == "float32" else 2
        # the logits, once more in the backward pass (they are not kept), and the two products of their gradient
        return {"bytes": size * float(d) * (N + B) * (2 if step else 1) + 16.0 * B, "flops": (8.0 if step else 2.0) * B * N * d}
    if case["kind"] == "eq4":
        d, m, b = case["d"], case["m"], case["b"]
        return {"bytes": 4.0 * (B * m * b + 2 * B * d + 2 * b * d), "flops": 4.0 * B * b * d}
    N, d, group = case["N"], case["d"], case["group"]
    return {"bytes": float(N) * (d / 2 + 2.0 * d / group) + 4.0 * B * (d + N), "flops": 2.0 * B * N * d}
