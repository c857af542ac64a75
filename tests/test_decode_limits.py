"""Sizes at the end of what the decode loop's calls take, without a GPU."""
import pytest

from paper_2609_37581_amd import trevs
from test_cache_abi import _cache, ptr, ref
from test_decode_abi import _evict

MOST = (1 << 31) - 1 - 1024


@pytest.mark.parametrize("B,n_keep,taken", [
    (1, MOST, True), (1, MOST + 1, False), (1, (1 << 31) - 1, False), (2, MOST // 2, True), (2, MOST // 2 + 1, False),
    (1024, MOST // 1024, True), (1024, MOST // 1024 + 1, False),
])
def test_evict_list_of_kept_tokens_stays_in_32_bits(B, n_keep, taken):
    """A workgroup's threads walk the list [B,n_keep] in steps of up to 1024: no place may pass 2^31 - 1."""
    L = trevs.lib()
    c, a = _cache(n_slots=2048), _evict(B=B, n_keep=n_keep, slots=ptr(25))
    assert (L.trevs_kv8_evict_workspace_size(ref(c), ref(a)) > 0) == taken
    assert L.trevs_kv8_evict(ref(c), ref(a), None, 0, None) == (3 if taken else 2)  # (no workspace: nothing is launched)
