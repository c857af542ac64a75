"""The decode loop's C ABI without a GPU: struct mirrors and the refusals that
come before any HIP call."""
import ctypes

import pytest
import torch

from paper_2609_37581_amd import trevs
from test_cache_abi import BAD_CACHE, _cache, _rope, fill, ptr, ref


def _norm(rope=None, **kw):
    a = trevs.NormRopeArgs()
    a.struct_size = ctypes.sizeof(a)
    fill(a, eps=1e-6, weight_offset=1.0, weight_dtype=trevs.TREVS_BF16, q_weight=ptr(6), k_weight=ptr(7))
    a.rope = _rope(**(rope or {}))
    return fill(a, **kw)


def _weights(**kw):
    a = trevs.Kv8WeightsArgs()
    a.struct_size = ctypes.sizeof(a)
    return fill(fill(a, B=8, T_max=3, H_q=28, dtype=trevs.TREVS_BF16, causal=1, scale=0.1, decay=1.0, q=ptr(20),
                     lse=ptr(21), score=ptr(22)), **kw)


def _evict(**kw):
    a = trevs.Kv8EvictArgs()
    a.struct_size = ctypes.sizeof(a)
    return fill(fill(a, B=8, n_keep=100, n_first=4, n_last=20, score=ptr(20), n_evicted=ptr(21), kept_idx=ptr(22)), **kw)


def _beam(**kw):
    a = trevs.BeamSelectArgs()
    a.struct_size = ctypes.sizeof(a)
    return fill(fill(a, B=3, W=4, V=1000, n_out=8, dtype=trevs.TREVS_BF16, logits=ptr(20), score=ptr(21),
                     score_out=ptr(22), parent=ptr(23), token=ptr(24)), **kw)


def test_struct_mirror_sizes():
    L = trevs.lib()
    for size, struct in ((L.trevs_norm_rope_args_size, trevs.NormRopeArgs),
                         (L.trevs_kv8_weights_args_size, trevs.Kv8WeightsArgs),
                         (L.trevs_kv8_evict_args_size, trevs.Kv8EvictArgs),
                         (L.trevs_beam_select_args_size, trevs.BeamSelectArgs)):
        assert size() == ctypes.sizeof(struct)


@pytest.mark.parametrize("bad,rope,code", [
    (dict(struct_size=8), {}, 1), (dict(eps=0.0), {}, 1), (dict(eps=-1e-6), {}, 1), (dict(eps=1e-40), {}, 1),
    (dict(eps=float("nan")), {}, 1), (dict(eps=float("inf")), {}, 1), (dict(weight_offset=float("inf")), {}, 1),
    (dict(weight_dtype=2), {}, 1), (dict(per_head=2), {}, 1), (dict(q_weight=ptr(6, 8)), {}, 1),
    (dict(k_weight=ptr(7, 2)), {}, 1), (dict(q_weight=ptr(4)), {}, 1),                  # weights in the output
    (dict(k_weight=ptr(5, 2 * 100 * 4 * 128 * 2 - 16)), {}, 1), (dict(per_head=1, k_weight=ptr(4, -512)), {}, 1),
    ({}, dict(struct_size=8), 1), ({}, dict(inverse=1), 1), ({}, dict(rot_dim=120), 1), ({}, dict(q=None), 1),
    ({}, dict(q_out=ptr(2, 256)), 1), ({}, dict(d_head=96, rot_dim=96, section=[16, 16, 16]), 2),
])
def test_norm_rope_rejects_before_launch(bad, rope, code):
    assert trevs.lib().trevs_norm_rope(ref(_norm(rope, **bad)), None) == code


@pytest.mark.parametrize("bad,code", BAD_CACHE)
def test_every_entry_point_rejects_a_bad_cache(bad, code):
    L = trevs.lib()
    c = ref(_cache(**bad))
    assert L.trevs_kv8_weights_workspace_size(c, ref(_weights())) == 0
    assert L.trevs_kv8_weights(c, ref(_weights()), None, 0, None) == code
    assert L.trevs_kv8_evict_workspace_size(c, ref(_evict())) == 0
    assert L.trevs_kv8_evict(c, ref(_evict()), None, 0, None) == code
    assert L.trevs_pages_reorder(c, 2, 4, ptr(30), ptr(31), None, None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(struct_size=8), 1), (dict(B=0), 1), (dict(T_max=0), 1), (dict(H_q=30), 1), (dict(layer=2), 1),
    (dict(causal=2), 1), (dict(kv_max=321), 1), (dict(kv_max=-1), 1), (dict(scale=0.0), 1),
    (dict(scale=float("nan")), 1), (dict(decay=-0.5), 1), (dict(decay=float("inf")), 1), (dict(dtype=5), 1),
    (dict(B=9), 1), (dict(B=9, slots=ptr(25)), 1), (dict(q=None), 1), (dict(lse=None), 1), (dict(score=None), 1),
    (dict(q=ptr(20, 8)), 1), (dict(lse=ptr(21, 2)), 1), (dict(score=ptr(22, 2)), 1), (dict(q_ld=28 * 128 + 4), 1),
    (dict(score=ptr(20, 256)), 1), (dict(score=ptr(21)), 1), (dict(score=ptr(14)), 1), (dict(q_len=ptr(22)), 1),
    (dict(slots=ptr(22, 64)), 1), (dict(H_q=1028), 2), (dict(B=8, T_max=1 << 27), 2),
])
def test_weights_reject_before_launch(bad, code):
    L = trevs.lib()
    assert L.trevs_kv8_weights_workspace_size(ref(_cache()), ref(_weights(**bad))) == 0
    assert L.trevs_kv8_weights(ref(_cache()), ref(_weights(**bad)), ptr(50), 1 << 40, None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(struct_size=8), 1), (dict(B=0), 1), (dict(n_keep=0), 1), (dict(n_first=-1), 1), (dict(n_last=-1), 1),
    (dict(n_first=60, n_last=41), 1), (dict(n_first=1 << 30, n_last=1 << 30, n_keep=100), 1), (dict(B=9), 1),
    (dict(score=None), 1), (dict(n_evicted=None), 1), (dict(kept_idx=None), 1), (dict(kept_idx=ptr(22, 2)), 1),
    (dict(keep=ptr(25, 1)), 1), (dict(slots=ptr(25, 2)), 1), (dict(kept_idx=ptr(20)), 1), (dict(keep=ptr(21)), 1),
    (dict(n_evicted=ptr(15)), 1), (dict(score=ptr(16)), 1), (dict(slots=ptr(14)), 1),
    (dict(B=1025, slots=ptr(25)), 2), (dict(B=1024, slots=ptr(25), n_keep=1 << 22), 2),
])
def test_evict_rejects_before_launch(bad, code):
    L = trevs.lib()
    assert L.trevs_kv8_evict_workspace_size(ref(_cache()), ref(_evict(**bad))) == 0
    assert L.trevs_kv8_evict(ref(_cache()), ref(_evict(**bad)), ptr(50), 1 << 40, None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(struct_size=8), 1), (dict(B=0), 1), (dict(W=0), 1), (dict(V=0), 1), (dict(n_out=0), 1), (dict(eos=-1), 1),
    (dict(eos=1000), 1), (dict(dtype=2), 1), (dict(logits_ld=999), 1), (dict(logits_ld=-1), 1), (dict(logits=None), 1),
    (dict(logits=ptr(20, 1)), 1), (dict(dtype=trevs.TREVS_F32, logits=ptr(20, 2)), 1), (dict(score=None), 1),
    (dict(done=ptr(25, 2)), 1), (dict(score_out=None), 1), (dict(parent=ptr(23, 2)), 1), (dict(token=None), 1),
    (dict(token=ptr(23, 32)), 1), (dict(parent=ptr(20, 64)), 1), (dict(done=ptr(24)), 1), (dict(W=65), 2),
    (dict(n_out=65), 2), (dict(W=64, V=1 << 26), 2), (dict(W=1, V=(1 << 31) - 2000), 2),
    (dict(B=1 << 22, W=64, V=100000), 2),
    (dict(logits_ld=1 << 32), 2),
])
def test_beam_select_rejects_before_launch(bad, code):
    L = trevs.lib()
    assert L.trevs_beam_select_workspace_size(ref(_beam(**bad))) == 0
    assert L.trevs_beam_select(ref(_beam(**bad)), ptr(50), 1 << 40, None) == code


def test_reorder_rejects_before_launch():
    L = trevs.lib()
    c, slots, parent, score = ref(_cache()), ptr(30), ptr(31), ptr(32)
    assert L.trevs_pages_reorder(c, 0, 4, slots, parent, score, None) == 1
    assert L.trevs_pages_reorder(c, 2, 0, slots, parent, score, None) == 1
    assert L.trevs_pages_reorder(c, 2, 4, slots, None, score, None) == 1
    assert L.trevs_pages_reorder(c, 3, 3, None, parent, score, None) == 1  # more than the slots there are
    assert L.trevs_pages_reorder(c, 2, 4, slots + 2, parent, score, None) == 1
    assert L.trevs_pages_reorder(c, 2, 4, slots, parent + 1, score, None) == 1
    assert L.trevs_pages_reorder(c, 2, 4, slots, parent, score + 2, None) == 1
    assert L.trevs_pages_reorder(c, 2, 4, slots, score + 64, score, None) == 1
    assert L.trevs_pages_reorder(c, 2, 4, ptr(14), parent, None, None) == 1
    assert L.trevs_pages_reorder(c, 2, 4, slots, ptr(15), None, None) == 1
    assert L.trevs_pages_reorder(c, 2, 4, slots, parent, ptr(10), None) == 1
    assert L.trevs_pages_reorder(c, 1, 65, slots, parent, None, None) == 2
    assert L.trevs_pages_reorder(c, 257, 4, slots, parent, None, None) == 2


def test_workspace_errors():
    L = trevs.lib()
    c = _cache()
    for args, size, call in ((_weights(T_max=100), L.trevs_kv8_weights_workspace_size, L.trevs_kv8_weights),
                             (_weights(), L.trevs_kv8_weights_workspace_size, L.trevs_kv8_weights),
                             (_evict(), L.trevs_kv8_evict_workspace_size, L.trevs_kv8_evict)):
        need = size(ref(c), ref(args))
        assert need > 0
        assert call(ref(c), ref(args), None, need, None) == 3
        assert call(ref(c), ref(args), ptr(50), need - 1, None) == 3
        assert call(ref(c), ref(args), ptr(50, 16), need, None) == 3
    a = _beam()
    need = L.trevs_beam_select_workspace_size(ref(a))
    assert need > 0
    assert L.trevs_beam_select(ref(a), None, need, None) == 3
    assert L.trevs_beam_select(ref(a), ptr(50), need - 1, None) == 3
    assert L.trevs_beam_select(ref(a), ptr(50, 16), need, None) == 3


def test_weights_workspace_stays_small_without_a_bound():
    """64 MB for any call whose scores are less than that."""
    c = _cache(n_slots=64, max_pages=20000)
    for B, H_q in ((1, 4), (3, 32), (40, 8)):
        need = trevs.lib().trevs_kv8_weights_workspace_size(ref(c), ref(_weights(B=B, H_q=H_q, T_max=500)))
        assert 0 < need <= 64 << 20


def test_binding_refuses_tensors_on_the_host():
    with pytest.raises(ValueError):
        trevs.BeamSelect(torch.zeros(1, 2, 8), torch.zeros(1, 2), n_out=2)
    with pytest.raises(ValueError):
        trevs.BeamSelect(torch.zeros(2, 8), torch.zeros(1, 2), n_out=2)
    q = torch.zeros(1, 2, 4, 64)
    with pytest.raises(ValueError):
        trevs.NormRope(q, None, torch.zeros(1, 1, 2, dtype=torch.int64), freqs=torch.zeros(32, dtype=torch.float64))
