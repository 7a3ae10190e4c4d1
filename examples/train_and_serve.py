"""Train both scoring heads on a synthetic catalogue and rank it with what they learned.

    python examples/train_and_serve.py [--items N] [--positions B] [--steps K]

Positions stand for what a sequence model returns at the end of its users' histories: here their embeddings are learned
directly, beside the items', so that each position comes to rank its own target first.

  by sub-ids       Eq. 4's tables, the softmax cross entropy of the whole catalogue by Eq. 5, its gradient with respect to the
                   tables and Eq. 4's gradients; then the top K by pq_score_topk()
  default scorer   the same loss by W phi in bfloat16, with float32 parameters beside; then W in four bits, its scores and
                   their top K
  distillation     the trained default scorer's likeliest items, with their log-probabilities, are the lists that a second head
                   by sub-ids learns from; then how likely it takes each target to be, and how sure it is
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2408_09992_amd as pq  # noqa: E402
from paper_2408_09992_amd import workloads  # noqa: E402


def found(ids, targets):
    """Share of the positions whose target is among their ids."""
    return (ids == targets[:, None]).any(1).float().mean().item()


def sub_ids(N, targets, d, m, b, steps, K, log):
    B = targets.numel()
    codes = torch.from_numpy(workloads.codes_uniform(N, m, b, seed=1)).cuda()
    torch.manual_seed(2)
    queries = torch.randn(B, d, device="cuda").div_(d ** 0.25).requires_grad_()
    centroids = torch.randn(m, b, d // m, device="cuda").div_(d ** 0.25).requires_grad_()
    adam = torch.optim.Adam([queries, centroids], lr=0.01)
    share = torch.full((B,), 1.0 / B, device="cuda")              # the objective is the positions' mean
    losses = []
    for step in range(steps):
        S = pq.pq_subitem_scores(queries.detach(), centroids.detach())
        loss, lse = pq.pq_cross_entropy(codes, S, targets)
        dS = pq.pq_cross_entropy_backward(codes, S, targets, lse, share)
        queries.grad, centroids.grad = pq.pq_subitem_scores_backward(dS, queries.detach(), centroids.detach())
        adam.step()
        losses.append(loss.mean().item())
        if step % 10 == 0:
            log(f"by sub-ids      step {step:4d}  loss {losses[-1]:.4f}")
    ids, _ = pq.pq_score_topk(codes, pq.pq_subitem_scores(queries.detach(), centroids.detach()), K)
    return losses, found(ids, targets)


def default_scorer(N, targets, d, steps, K, log):
    B = targets.numel()
    torch.manual_seed(3)
    queries = torch.randn(B, d, device="cuda").div_(d ** 0.25).requires_grad_()
    W = torch.randn(N, d, device="cuda").div_(d ** 0.25).requires_grad_()
    adam = torch.optim.Adam([queries, W], lr=0.01)
    share = torch.full((B,), 1.0 / B, device="cuda")
    losses = []
    for step in range(steps):
        q16, w16 = queries.detach().bfloat16(), W.detach().bfloat16()
        loss, lse = pq.pq_default_cross_entropy(w16, q16, targets)
        dq, dw = pq.pq_default_cross_entropy_backward(w16, q16, targets, lse, share)
        queries.grad, W.grad = dq.float(), dw.float()
        adam.step()
        losses.append(loss.mean().item())
        if step % 10 == 0:
            log(f"default scorer  step {step:4d}  loss {losses[-1]:.4f}")
    packed, scales = pq.pq_quantise_items(W.detach(), 64)
    ids4, _ = pq.pq_topk_scores(pq.pq_default_scores_q4(packed, scales, queries.detach()), K, N)
    ids, _ = pq.pq_topk_scores(pq.pq_default_scores(W.detach(), queries.detach()), K, N)
    return losses, found(ids4, targets), found(ids, targets), W.detach(), queries.detach()


def distillation(teacher_W, teacher_queries, targets, d, m, b, steps, K, T, log):
    """A head by sub-ids learns what the default scorer W phi would answer; returns the losses, the share of positions whose likeliest item is
    the teacher's, and each target's log-probability and the entropy as the student has them."""
    N, B = teacher_W.shape[0], targets.numel()
    _, _, _, teacher_items, teacher_scores = pq.pq_default_log_probs(teacher_W, teacher_queries, None, K)
    codes = torch.from_numpy(workloads.codes_uniform(N, m, b, seed=1)).cuda()
    torch.manual_seed(5)
    queries = torch.randn(B, d, device="cuda").div_(d ** 0.25).requires_grad_()
    centroids = torch.randn(m, b, d // m, device="cuda").div_(d ** 0.25).requires_grad_()
    adam = torch.optim.Adam([queries, centroids], lr=0.01)
    share = torch.full((B,), 1.0 / B, device="cuda")
    losses = []
    for step in range(steps):
        S = pq.pq_subitem_scores(queries.detach(), centroids.detach())
        loss, lse = pq.pq_distillation(codes, S, teacher_items, teacher_scores, T)
        dS = pq.pq_distillation_backward(codes, S, teacher_items, teacher_scores, lse, share, T)
        queries.grad, centroids.grad = pq.pq_subitem_scores_backward(dS, queries.detach(), centroids.detach())
        adam.step()
        losses.append(loss.mean().item())
        if step % 10 == 0:
            log(f"distillation    step {step:4d}  loss {losses[-1]:.4f}")
    S = pq.pq_subitem_scores(queries.detach(), centroids.detach())
    log_probs, entropy, _, likeliest, _ = pq.pq_log_probs(codes, S, targets[:, None], 1)
    return losses, (likeliest[:, 0] == teacher_items[:, 0]).float().mean().item(), log_probs[:, 0], entropy


def main(items=100_000, positions=512, steps=100, d=128, m=8, b=256, K=10, log=print):
    targets = torch.from_numpy(workloads.candidate_list(items, positions, seed=4)).to(torch.int32).cuda()
    log(f"{items} items, {positions} positions: untrained loss about log N = {math.log(items):.2f}")
    losses, hits = sub_ids(items, targets, d, m, b, steps, K, log)
    log(f"by sub-ids      loss {losses[0]:.4f} -> {losses[-1]:.4f}; targets among the top {K}: {hits:.3f}")
    dense, hits4, hits32, W, queries = default_scorer(items, targets, d, steps, K, log)
    log(f"default scorer  loss {dense[0]:.4f} -> {dense[-1]:.4f}; targets among the top {K}: {hits4:.3f} from four bits, {hits32:.3f} in float32")
    taught, alike, log_probs, entropy = distillation(W, queries, targets, d, m, b, steps, K, 2.0, log)
    log(f"distillation    loss {taught[0]:.4f} -> {taught[-1]:.4f}; the teacher's first item first: {alike:.3f}; log-probability of the targets "
        f"{log_probs.mean().item():.3f}, entropy {entropy.mean().item():.3f}")
    return dict(sub_ids=losses, sub_ids_found=hits, default=dense, default_found=hits32, four_bits_found=hits4, distillation=taught,
                distillation_alike=alike, log_probs=log_probs, entropy=entropy)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--items", type=int, default=100_000)
    ap.add_argument("--positions", type=int, default=512)
    ap.add_argument("--steps", type=int, default=100)
    args = ap.parse_args()
    main(args.items, args.positions, args.steps)
