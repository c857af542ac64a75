"""The serving cache's C ABI without a GPU: struct mirrors, the frequencies
(a host function), and the refusals that come before any HIP call."""
import ctypes

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2609_37581_amd import trevs

BASE = 1 << 40


def ptr(i, off=0):
    return BASE + (i << 36) + off


def fill(a, **kw):
    for k, v in kw.items():
        if isinstance(v, (list, tuple)):
            for i, x in enumerate(v):
                getattr(a, k)[i] = x
        else:
            setattr(a, k, v)
    return a


def _rope(**kw):
    a = trevs.RopeArgs()
    a.struct_size = ctypes.sizeof(a)
    fill(a, B=2, S=100, H_q=28, H_k=4, d_head=128, rot_dim=128, n_pos=3, section=[16, 24, 24], attn_factor=1.0,
         dtype=trevs.TREVS_BF16, freqs=ptr(0), pos=ptr(1), q=ptr(2), k=ptr(3), q_out=ptr(4), k_out=ptr(5))
    return fill(a, **kw)


def _cache(**kw):
    c = trevs.Kv8CacheArgs()
    c.struct_size = ctypes.sizeof(c)
    fill(c, n_layers=2, n_pages=64, page_tokens=16, H_kv=4, d_head=128, n_slots=8, max_pages=20, k=ptr(10), v=ptr(11),
         k_scale=ptr(12), v_scale=ptr(13), table=ptr(14), len=ptr(15), ref=ptr(16))
    return fill(c, **kw)


def _write(**kw):
    a = trevs.Kv8WriteArgs()
    a.struct_size = ctypes.sizeof(a)
    return fill(fill(a, B=8, T_max=33, dtype=trevs.TREVS_BF16, k=ptr(20), v=ptr(21)), **kw)


def _attn(**kw):
    a = trevs.Kv8AttentionArgs()
    a.struct_size = ctypes.sizeof(a)
    return fill(fill(a, B=8, T_max=3, H_q=28, dtype=trevs.TREVS_BF16, causal=1, scale=0.1, q=ptr(20), out=ptr(21)), **kw)


def _compact(**kw):
    a = trevs.Kv8CompactArgs()
    a.struct_size = ctypes.sizeof(a)
    return fill(fill(a, B=3, P=5, K_in=100, n_kept=30, kept_idx=ptr(20), src_slots=ptr(21), dst_slots=ptr(22)), **kw)


def ref(x):
    return ctypes.byref(x)


def test_struct_mirror_sizes():
    L = trevs.lib()
    for size, struct in ((L.trevs_rope_args_size, trevs.RopeArgs), (L.trevs_kv8_cache_size, trevs.Kv8CacheArgs),
                         (L.trevs_kv8_write_args_size, trevs.Kv8WriteArgs),
                         (L.trevs_kv8_attention_args_size, trevs.Kv8AttentionArgs),
                         (L.trevs_kv8_compact_args_size, trevs.Kv8CompactArgs)):
        assert size() == ctypes.sizeof(struct)


@pytest.mark.parametrize("kw", [
    dict(rot_dim=128), dict(rot_dim=64, base=500000.0, scaling="linear", factor=4.0),
    dict(rot_dim=128, base=1e6, scaling="parts", factor=8.0, original_len=8192),
    dict(rot_dim=48, scaling="parts", factor=2.5, original_len=4096, beta_fast=16.0, beta_slow=2.0),
])
def test_rope_frequencies(kw):
    got = trevs.rope_frequencies(**kw).numpy()
    # a power, a division or two and a blend of doubles: each within an ulp or so
    assert np.allclose(got, co.rope_frequencies(**kw), rtol=1e-14, atol=0)


@pytest.mark.parametrize("kw", [
    dict(rot_dim=15), dict(rot_dim=0), dict(rot_dim=16, base=0.0), dict(rot_dim=16, base=float("nan")),
    dict(rot_dim=16, scaling="linear", factor=0.0), dict(rot_dim=16, scaling="parts", factor=2.0),
    dict(rot_dim=16, scaling="parts", factor=2.0, original_len=100, beta_fast=1.0, beta_slow=1.0),
    dict(rot_dim=16, scaling="parts", factor=float("inf"), original_len=100),
])
def test_rope_frequencies_refusals(kw):
    with pytest.raises(trevs.TrevsError):
        trevs.rope_frequencies(**kw)
    with pytest.raises(ValueError):
        trevs.rope_frequencies(16, scaling="other")


@pytest.mark.parametrize("bad,code", [
    (dict(struct_size=8), 1), (dict(B=0), 1), (dict(S=0), 1), (dict(H_q=0, H_k=0), 1), (dict(H_q=-1), 1),
    (dict(rot_dim=120), 1), (dict(rot_dim=144), 1), (dict(rot_dim=0), 1), (dict(section=[16, 24, 23]), 1),
    (dict(section=[70, -30, 24]), 1), (dict(n_pos=0), 1), (dict(n_pos=5), 1), (dict(interleaved=2), 1),
    (dict(inverse=-1), 1), (dict(dtype=2), 1), (dict(attn_factor=float("inf")), 1), (dict(freqs=None), 1),
    (dict(pos=ptr(1, 4)), 1), (dict(q=None), 1), (dict(k_out=ptr(5, 8)), 1), (dict(q_ld=28 * 128 - 8), 1),
    (dict(q_ld=28 * 128 + 4), 1), (dict(q_out=ptr(2, 256)), 1), (dict(q_out=ptr(2), q_out_ld=28 * 128 + 8), 1),
    (dict(k_out=ptr(2, 1024)), 1), (dict(q_out=ptr(5)), 1), (dict(q_out=ptr(1)), 1), (dict(d_head=96, rot_dim=96, section=[16, 16, 16]), 2),
    (dict(B=1 << 20, S=1 << 12), 2), (dict(H_q=2000), 2),
    # slices of one buffer that do meet
    (dict(q=ptr(2), k=ptr(2, 27 * 256), q_ld=36 * 128, k_ld=36 * 128, q_out=ptr(2), k_out=ptr(2, 27 * 256),
          q_out_ld=36 * 128, k_out_ld=36 * 128), 1),
])
def test_rope_rejects_before_launch(bad, code):
    assert trevs.lib().trevs_rope(ref(_rope(**bad)), None) == code


BAD_CACHE = [
    (dict(struct_size=8), 1), (dict(n_layers=0), 1), (dict(n_pages=0), 1), (dict(H_kv=0), 1), (dict(n_slots=0), 1),
    (dict(max_pages=0), 1), (dict(k=None), 1), (dict(v=ptr(11, 8)), 1), (dict(k_scale=ptr(12, 2)), 1),
    (dict(table=None), 1), (dict(len=ptr(15, 1)), 1), (dict(ref=None), 1), (dict(d_head=96), 2),
    (dict(page_tokens=48), 2), (dict(page_tokens=128), 2), (dict(max_pages=1 << 27), 2), (dict(H_kv=2000), 2),
]


@pytest.mark.parametrize("bad,code", BAD_CACHE)
def test_every_cache_entry_point_rejects_a_bad_cache(bad, code):
    L = trevs.lib()
    c = _cache(**bad)
    lists = [ptr(30 + i) for i in range(5)]
    assert L.trevs_pages_reserve(ref(c), 3, *lists, None) == code
    assert L.trevs_pages_fork(ref(c), 3, *lists[:4], None) == code
    assert L.trevs_pages_free(ref(c), 3, *lists[:2], None) == code
    assert L.trevs_kv8_copy_pages(ref(c), 3, *lists[:2], None) == code
    assert L.trevs_kv8_write(ref(c), ref(_write()), None) == code
    assert L.trevs_kv8_attention_workspace_size(ref(c), ref(_attn())) == 0
    assert L.trevs_kv8_attention(ref(c), ref(_attn()), None, 0, None) == code
    assert L.trevs_kv8_compact(ref(c), ref(_compact()), None) == code


def test_page_operations_reject_before_launch():
    L = trevs.lib()
    c = ref(_cache())
    a, b, d, e, f = [ptr(30 + i) for i in range(5)]
    assert L.trevs_pages_reserve(c, 0, a, b, d, e, f, None) == 1
    assert L.trevs_pages_reserve(c, 9, None, b, d, e, f, None) == 1     # more than the slots there are
    assert L.trevs_pages_reserve(c, 1025, a, b, d, e, f, None) == 2
    assert L.trevs_pages_reserve(c, 3, a, None, d, e, f, None) == 1
    assert L.trevs_pages_reserve(c, 3, a, b, d, e, None, None) == 1
    assert L.trevs_pages_reserve(c, 3, a, b, b, e, f, None) == 1        # granted on n_new
    assert L.trevs_pages_reserve(c, 3, a, b, d, e, e + 8, None) == 1    # outputs meet
    assert L.trevs_pages_reserve(c, 3, a, b + 2, d, e, f, None) == 1
    assert L.trevs_pages_reserve(c, 3, ptr(15), b, d, e, f, None) == 1  # the lengths as the list of slots
    assert L.trevs_pages_fork(c, 3, None, b, None, d, None) == 1
    assert L.trevs_pages_fork(c, 3, a, None, None, d, None) == 1
    assert L.trevs_pages_fork(c, 3, a, b, None, None, None) == 1
    assert L.trevs_pages_fork(c, 3, a, b, None, a, None) == 1
    assert L.trevs_pages_fork(c, 1025, a, b, None, d, None) == 2
    assert L.trevs_pages_free(c, 9, None, None, None) == 1
    assert L.trevs_pages_free(c, 3, a, b + 1, None) == 1
    assert L.trevs_pages_free(c, 3, a, ptr(14), None) == 1
    assert L.trevs_kv8_copy_pages(c, 0, a, b, None) == 1
    assert L.trevs_kv8_copy_pages(c, 3, a, None, None) == 1
    assert L.trevs_kv8_copy_pages(c, 3, ptr(16), b, None) == 1


@pytest.mark.parametrize("bad,code", [
    (dict(struct_size=8), 1), (dict(B=0), 1), (dict(T_max=0), 1), (dict(layer=2), 1), (dict(layer=-1), 1),
    (dict(dtype=5), 1), (dict(B=9), 1), (dict(k=None), 1), (dict(v=ptr(21, 8)), 1), (dict(k_ld=511), 1),
    (dict(v_ld=516), 1), (dict(n_new=ptr(22, 2)), 1), (dict(k=ptr(10, 4096)), 1), (dict(n_new=ptr(15)), 1),
    (dict(slots=ptr(14, 4)), 1), (dict(B=8, T_max=1 << 29), 2),
])
def test_write_rejects_before_launch(bad, code):
    assert trevs.lib().trevs_kv8_write(ref(_cache()), ref(_write(**bad)), None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(struct_size=8), 1), (dict(B=0), 1), (dict(T_max=0), 1), (dict(H_q=30), 1), (dict(layer=2), 1),
    (dict(causal=2), 1), (dict(kv_max=321), 1), (dict(kv_max=-1), 1), (dict(scale=0.0), 1),
    (dict(scale=float("nan")), 1), (dict(dtype=5), 1), (dict(B=9), 1), (dict(q=None), 1), (dict(out=ptr(21, 8)), 1),
    (dict(out=ptr(20, 256)), 1), (dict(out=ptr(10, 256)), 1), (dict(lse=ptr(21, 64)), 1), (dict(lse=ptr(15)), 1),
    (dict(q_ld=28 * 128 + 4), 1), (dict(q_len=ptr(21)), 1), (dict(H_q=1028), 2), (dict(B=8, T_max=1 << 27), 2),
])
def test_attention_rejects_before_launch(bad, code):
    L = trevs.lib()
    assert L.trevs_kv8_attention_workspace_size(ref(_cache()), ref(_attn(**bad))) == 0
    assert L.trevs_kv8_attention(ref(_cache()), ref(_attn(**bad)), ptr(50), 1 << 40, None) == code


def test_attention_workspace_errors():
    L = trevs.lib()
    c, a = _cache(), _attn()
    need = L.trevs_kv8_attention_workspace_size(ref(c), ref(a))
    assert need > 0
    assert L.trevs_kv8_attention(ref(c), ref(a), None, need, None) == 3
    assert L.trevs_kv8_attention(ref(c), ref(a), ptr(50), need - 1, None) == 3
    assert L.trevs_kv8_attention(ref(c), ref(a), ptr(50, 16), need, None) == 3


@pytest.mark.parametrize("bad,code", [
    (dict(struct_size=8), 1), (dict(B=0), 1), (dict(P=-1), 1), (dict(K_in=0), 1), (dict(n_kept=101), 1),
    (dict(n_kept=0), 1), (dict(kept_idx=None), 1), (dict(src_slots=ptr(21, 2)), 1), (dict(dst_slots=None), 1),
    (dict(P=300), 1), (dict(kept_idx=ptr(14)), 1), (dict(B=1 << 28, n_kept=1), 2),
])
def test_compact_rejects_before_launch(bad, code):
    assert trevs.lib().trevs_kv8_compact(ref(_cache()), ref(_compact(**bad)), None) == code
