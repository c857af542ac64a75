"""Calls over tables far longer than their sequences."""
import numpy as np
import pytest
import torch

from paper_2609_37581_amd import trevs
from test_gpu_cache import check_contents, check_table, dev, device_cache, model
from test_gpu_cache_workspace import lengthened

pytestmark = pytest.mark.gpu


def run_compact(m, P, K_in, K, src, dst, seed=0):
    rng = np.random.default_rng(seed)
    c = device_cache(m)
    kept = np.sort(np.argsort(rng.random((len(src), K_in)), 1)[:, :K], 1)
    trevs.kv8_compact(c, dev(kept), dev(src), dev(dst), P=P, K_in=K_in)
    m.compact(kept, src, dst, P, K_in)
    check_contents(c, m)
    check_table(c, m)


@pytest.mark.parametrize("page,d", [(16, 64), (32, 128), (64, 256)])
@pytest.mark.parametrize("batch", [3, 2048])
def test_compact_sequences_longer_than_the_launch(page, d, batch):
    """A few kept rows of sequences with a long rest: with many samples (most
    of them skipped) a workgroup takes several blocks of a sequence, with few one."""
    P, K_in, K = 3, 90, 5
    lens = [P + K_in + 17 * page + 5, P + K_in + 1, P + K_in + 40 * page]
    m = lengthened(model(np.random.default_rng(page), lens + [n - K_in + K for n in lens], page, 2, d, n_layers=2), 1000)
    m.table[3][2] = -1  # a destination page that is not there is passed over
    src, dst = [-1] * batch, [-1] * batch
    for i, at in enumerate((0, batch // 2, batch - 1)):
        src[at], dst[at] = i, 3 + i
    run_compact(m, P, K_in, K, src, dst)


def test_compact_under_a_very_long_table():
    """Workgroups for every place of this table (a million tokens, 16 layers, 128
    samples, 8 heads) would be more than a launch can have."""
    P, K_in, K = 5, 200, 60
    lens = [P + K_in + 30, P + K_in + 3]
    m = lengthened(model(np.random.default_rng(2), lens + [n - K_in + K for n in lens], 64, 8, 64, n_layers=16), 16384)
    src, dst = [-1] * 128, [-1] * 128
    src[0], dst[0], src[127], dst[127] = 0, 2, 1, 3
    run_compact(m, P, K_in, K, src, dst)
