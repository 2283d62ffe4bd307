"""Tiered pooled-embedding lookup for MI355X (gfx950): HIP kernels behind the C
ABI of include/recmg.h, with a thin ctypes binding.

The lookup is the per-batch pooled embedding-bag gather that RecMG's caching and
prefetching decisions (arXiv 2511.08568) act on: full tables in pinned host
DRAM, a row cache in HBM, residency set between batches from caller-supplied
prefetch lists and caching bits.

Beside it, for tables that HBM holds and for training: token lookups with a scale,
the gradient of token and pooled lookups, the norm of gradients and clipping.
"""
from .binding import (  # noqa: F401
    EXPORTED,
    RecmgError,
    TieredEmbeddingCache,
    load_library,
    recmg_apply_placement,
    recmg_cache_destroy,
    recmg_cache_init,
    recmg_cache_init_static,
    recmg_config_t,
    recmg_embbag_forward,
    recmg_embedding_backward,
    recmg_embedding_backward_rows,
    recmg_embedding_forward,
    recmg_grad_clip,
    recmg_grad_norm,
    recmg_grad_norm_clip,
    recmg_last_error,
    recmg_query_embedding_workspace,
    recmg_query_grad_workspace,
    recmg_query_workspace,
    recmg_set_timing,
    recmg_stage_times,
    recmg_stats,
    recmg_stats_log,
    recmg_table_stats_t,
)

_EMBEDDING = ("embedding_forward", "embedding_backward", "embedding_backward_rows")
_GRADIENTS = ("GradientList", "grad_norm", "clip_grads", "clip_grad_norm")


def __getattr__(name):
    """The calls that take torch tensors: their modules import torch, which the C binding alone does not need."""
    import importlib
    if name not in _EMBEDDING + _GRADIENTS:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    value = getattr(importlib.import_module(".embedding" if name in _EMBEDDING else ".gradients", __name__), name)
    globals()[name] = value  # found without this function from now on
    return value
