"""Values that the decode loop's calls promise to keep apart, against the float64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import decode_oracle as do
from paper_2609_37581_amd import trevs
from test_gpu_cache import device_cache, host, model, storage
from test_gpu_decode import check_weights, scores_for

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]

# page, H_q, H_kv, d, T, lens, q_len; rows of a group from one to past a few stages of 32 and of 64, whole ones among them
FIRST_ROWS = [
    (16, 2, 2, 64, 1, [1, 40], None), (32, 4, 1, 128, 3, [3, 90], None), (64, 1, 1, 128, 70, [70, 70], None),
    (16, 2, 2, 64, 33, [33, 100], None), (32, 7, 1, 128, 25, [100, 25], None), (64, 3, 3, 128, 64, [64, 64], None),
    (32, 2, 1, 256, 40, [40, 300], None), (16, 6, 2, 64, 50, [50, 31], [47, 31]), (64, 1, 1, 128, 257, [257, 600], [257, 129]),
]


@pytest.mark.parametrize("shape", FIRST_ROWS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_weights_first_row_without_numbers(shape, dtype, value):
    """A first row that holds NaN or an infinity reaches the tokens that it sees and no others, whatever
    the number of rows, and the rows behind q_len may hold anything."""
    page, H_q, H_kv, d, T, lens, q_len = shape
    print(f"[first row] {shape} {dtype} {value}", flush=True)
    rng = np.random.default_rng(T + d)
    m = model(rng, lens, page, H_kv, d)
    c = device_cache(m)
    _, qs = storage(rng.normal(size=(2, T, H_q, d)), dtype)
    _, lse, _, _ = m.attention(qs, q_len=q_len)
    lse = np.where(np.isnan(lse), 9e9, lse)  # (rows past q_len: not read)
    qs[0, 0, ::H_q // H_kv, 3] = value
    lse[0, ::H_q // H_kv, 0] = math.nan
    rows = [T, T] if q_len is None else q_len
    for b in range(2):
        qs[b, rows[b]:] = math.nan
    q, qs = storage(qs, dtype)
    ld, ls = storage(lse, torch.float32)
    score, want = scores_for(m, c, rng)
    old = want.copy()
    bound = [np.nan_to_num(x) for x in do.weights(m, qs, ls, want, q_len=q_len)]
    assert np.isnan(want[0]).sum() == lens[0] - rows[0] + 1 and not np.isnan(want[1]).any()
    trevs.kv8_weights(c, q, ld, score, None if q_len is None else torch.tensor(q_len, dtype=torch.int32, device="cuda"))
    check_weights(host(score), want, *bound, 1.0, old)


@pytest.mark.parametrize("T,H_q,H_kv,d", [(50, 4, 2, 64), (40, 7, 1, 128), (33, 2, 1, 256)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_weights_rows_that_give_nothing(T, H_q, H_kv, d, dtype, value):
    """A row whose log-sum-exp is -inf gives nothing, whatever it holds."""
    check_rows_that_give_nothing(T, H_q, H_kv, d, dtype, value, 0)


@pytest.mark.parametrize("T,H_q,H_kv,d", [(1, 2, 1, 64), (3, 4, 2, 64), (1, 28, 4, 128), (2, 7, 1, 128), (4, 32, 4, 128),
                                          (3, 8, 1, 256), (1, 20, 10, 64)])
@pytest.mark.parametrize("max_pages", [0, 512])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_weights_few_rows_that_give_nothing(T, H_q, H_kv, d, max_pages, dtype, value):
    """The same for the kernels of few rows, under a short table and a long one."""
    check_rows_that_give_nothing(T, H_q, H_kv, d, dtype, value, max_pages)


def check_rows_that_give_nothing(T, H_q, H_kv, d, dtype, value, max_pages):
    rng = np.random.default_rng(T * d)
    m = model(rng, [120, T], 16, H_kv, d)
    if max_pages:
        m.table = [row + [-1] * (max_pages - len(row)) for row in m.table]
        m.max_pages = max_pages
    c = device_cache(m)
    x = rng.normal(size=(2, T, H_q, d))
    _, qs = storage(x, dtype)
    _, lse, _, _ = m.attention(qs)
    out = [(0, 0, 0), (0, T - 1, H_q - 1), (1, T // 2, 1), (1, 0, 0)]  # b, t, h
    for b, t, h in out:
        x[b, t, h, 5] = value
        qs[b, t, h] = 0.0  # (the oracle's)
        lse[b, h, t] = -math.inf
    q, _ = storage(x, dtype)
    ld, ls = storage(lse, torch.float32)
    score, want = scores_for(m, c, rng)
    old = want.copy()
    bound = do.weights(m, qs, ls, want)
    assert not np.isnan(want).any()
    trevs.kv8_weights(c, q, ld, score)
    check_weights(host(score), want, *bound, 1.0, old)
