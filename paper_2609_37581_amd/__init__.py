"""TReVS two-stage visual-token pruning on MI355X (gfx950).

The HIP library libtrevs.so (C ABI in include/trevs.h) does all the work;
`trevs` is its ctypes binding."""

from .trevs import (BeamSelect, Inllm, Kv8Attention, Kv8Cache, Kv8Compact, Kv8Copy,  # noqa: F401
                    Kv8Evict, Kv8Weights, Kv8Write, NormRope, PagesFork, PagesFree, PagesReorder,
                    PagesReserve, Prellm, Rope, TrevsError, beam_select, inllm_prune, keep_count,
                    kv8_attention, kv8_compact, kv8_copy, kv8_evict, kv8_scores, kv8_weights,
                    kv8_write, norm_rope, pages_fork, pages_free, pages_reorder, pages_reserve,
                    prellm_prune, rope, rope_frequencies, topk_select)
