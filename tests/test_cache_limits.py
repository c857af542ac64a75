"""The launch limits of the serving cache's entry points: sizes past them are
refused before anything is launched."""
import pytest

from paper_2609_37581_amd import trevs
from test_cache_abi import _cache, _compact, ref


@pytest.mark.parametrize("layers,B,H", [(1024, 16, 1024), (32, 1 << 17, 4), (2, 1 << 21, 4)])
def test_compact_launch_limit(layers, B, H):
    """A workgroup of up to 256 threads for each layer, sample and head: 2^32 threads and more."""
    c, a = _cache(n_layers=layers, H_kv=H, n_slots=B), _compact(B=B, K_in=4, n_kept=1)
    assert trevs.lib().trevs_kv8_compact(ref(c), ref(a), None) == 2
