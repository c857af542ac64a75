"""TReVS two-stage visual-token pruning on MI355X (gfx950).

The HIP library libtrevs.so (C ABI in include/trevs.h) does all the work;
`trevs` is its ctypes binding."""

from .trevs import (Inllm, Kv8Attention, Kv8Cache, Kv8Compact, Kv8Copy, Kv8Write,  # noqa: F401
                    PagesFork, PagesFree, PagesReserve, Prellm, Rope, TrevsError, inllm_prune,
                    keep_count, kv8_attention, kv8_compact, kv8_copy, kv8_write, pages_fork,
                    pages_free, pages_reserve, prellm_prune, rope, rope_frequencies, topk_select)
