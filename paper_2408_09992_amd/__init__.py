"""PQTopK scoring for sub-item-id (RecJPQ) recommendation models on MI355X (gfx950).

`workloads` draws the seeded synthetic inputs; the HIP path is reached through the names below, which load the
C-ABI library on first use and raise if it has not been built (there is no CPU fallback).
"""
from __future__ import annotations

__all__ = ["workloads", "pq_subitem_scores", "pq_score_topk", "pq_score_topk_workspace_bytes", "pq_score_topk_u16",
           "pq_score_topk_u16_workspace_bytes", "pq_score_topk_subset",
           "pq_score_topk_subset_workspace_bytes", "pq_topk_scores", "pq_topk_scores_workspace_bytes", "pq_recjpq_scores",
           "pq_reconstruct_items", "pq_default_scores", "pq_strerror", "pq_cross_entropy", "pq_cross_entropy_workspace_bytes",
           "pq_cross_entropy_backward", "pq_cross_entropy_backward_workspace_bytes", "pq_cross_entropy_u16",
           "pq_cross_entropy_u16_workspace_bytes", "pq_cross_entropy_u16_backward", "pq_cross_entropy_u16_backward_workspace_bytes",
           "pq_default_cross_entropy", "pq_default_cross_entropy_workspace_bytes", "pq_default_cross_entropy_backward",
           "pq_default_cross_entropy_backward_workspace_bytes",
           "pq_subitem_scores_backward", "pq_subitem_scores_backward_workspace_bytes", "pq_quantise_items", "pq_default_scores_q4",
           "pq_log_probs", "pq_log_probs_workspace_bytes", "pq_log_probs_u16", "pq_log_probs_u16_workspace_bytes", "pq_default_log_probs",
           "pq_default_log_probs_workspace_bytes", "pq_distillation", "pq_distillation_workspace_bytes", "pq_distillation_backward",
           "pq_distillation_backward_workspace_bytes", "pq_distillation_u16", "pq_distillation_u16_workspace_bytes",
           "pq_distillation_u16_backward", "pq_distillation_u16_backward_workspace_bytes", "pq_default_distillation",
           "pq_default_distillation_workspace_bytes", "pq_default_distillation_backward", "pq_default_distillation_backward_workspace_bytes"]


def __getattr__(name):
    if name in __all__[1:]:
        from . import binding
        globals()[name] = found = getattr(binding, name)       # (the next use finds it without coming here)
        return found
    if name in ("workloads", "binding", "build"):
        import importlib
        return importlib.import_module(f"{__name__}.{name}")
    raise AttributeError(name)
