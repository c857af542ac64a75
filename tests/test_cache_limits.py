"""The launch limits of the serving cache's entry points: sizes past them are
refused before anything is launched."""
import pytest

from paper_2609_37581_amd import trevs
from test_cache_abi import _attn, _cache, _compact, _rope, _write, ptr, ref


@pytest.mark.parametrize("layers,B,H", [(1024, 16, 1024), (32, 1 << 17, 4), (2, 1 << 21, 4)])
def test_compact_launch_limit(layers, B, H):
    """A workgroup of up to 256 threads for each layer, sample and head: 2^32 threads and more."""
    c, a = _cache(n_layers=layers, H_kv=H, n_slots=B), _compact(B=B, K_in=4, n_kept=1)
    assert trevs.lib().trevs_kv8_compact(ref(c), ref(a), None) == 2


def test_rope_launch_limit():
    """Two rows a workgroup of 256 threads at 256 turned values, eight at 64."""
    L = trevs.lib()
    kw = dict(H_q=1, H_k=0, n_pos=1, k=None, k_out=None)
    assert L.trevs_rope(ref(_rope(B=1 << 12, S=1 << 13, d_head=256, rot_dim=256, section=[128, 0, 0, 0], **kw)), None) == 2
    assert L.trevs_rope(ref(_rope(B=1 << 14, S=1 << 13, d_head=64, rot_dim=64, section=[32, 0, 0, 0], **kw)), None) == 2


def test_write_launch_limit():
    c = _cache(n_slots=1 << 20, max_pages=1 << 10, H_kv=16)
    assert trevs.lib().trevs_kv8_write(ref(c), ref(_write(B=1 << 20, T_max=1)), None) == 2
    assert trevs.lib().trevs_kv8_write(ref(c), ref(_write(B=1 << 12, T_max=4081)), None) == 2


@pytest.mark.parametrize("B,T,dtype", [(1 << 22, 1, trevs.TREVS_BF16), (1 << 16, 512, trevs.TREVS_F32)])
def test_attention_launch_limit(B, T, dtype):
    L = trevs.lib()
    c = _cache(n_slots=B, d_head=256)
    a = _attn(B=B, T_max=T, H_q=32 if T == 1 else 16, dtype=dtype, q=1 << 44, out=1 << 45)  # (512 GB each)
    assert L.trevs_kv8_attention_workspace_size(ref(c), ref(a)) == 0
    assert L.trevs_kv8_attention(ref(c), ref(a), ptr(50), 1 << 40, None) == 2


def test_copy_launch_limit():
    assert trevs.lib().trevs_kv8_copy_pages(ref(_cache(n_pages=1 << 24)), 1 << 24, ptr(30), ptr(31), None) == 2
