"""Pins of the decode loop's oracle: worked numbers, brute force and invariances."""
import math

import numpy as np

from oracle import cache_oracle as co
from oracle import decode_oracle as do


def small_cache(rng, lens, page=4, H=2, d=8, spare=12, n_layers=1, max_pages=8):
    need = [-(-n // page) for n in lens]
    m = co.CacheModel(sum(need) + spare, page, len(lens), max_pages, H, d, n_layers)
    order = rng.permutation(m.n_pages).tolist()
    for s, n in enumerate(need):
        m.table[s][:n] = [order.pop() for _ in range(n)]
        m.len[s] = lens[s]
        for p in m.table[s][:n]:
            m.ref[p] = 1
    for data, scale in ((m.k, m.k_scale), (m.v, m.v_scale)):
        x = rng.normal(size=data.shape)
        scale[:] = co.block_scale(np.abs(x).max((3, 4)))
        data[:] = co.e4m3(x / scale[..., None, None])
    return m


def test_norm_without_rotation_and_its_invariance():
    x = np.array([[[[3.0, 4.0] + [0.0] * 14]]])
    pos, f = np.zeros((1, 1, 1), np.int64), np.zeros(8)
    y, _ = do.norm_rope(x, None, 5.0, 0.0, pos, f, [8])
    assert np.allclose(y[0, 0, 0, :2], [3 / (5 / 4), 4 / (5 / 4)])  # root mean square 5 / sqrt(16)
    y, _ = do.norm_rope(x, np.ones(16), 1.0, 0.0, pos, f, [8])
    assert np.allclose(y[0, 0, 0, :2], [4.8, 6.4])
    rng = np.random.default_rng(0)
    x = rng.normal(size=(1, 3, 2, 16))
    pos, f = rng.integers(0, 99, (1, 1, 3)), co.rope_frequencies(16)
    a, _ = do.norm_rope(x, None, 0.0, 0.0, pos, f, [8])
    b, _ = do.norm_rope(1000 * x, None, 0.0, 0.0, pos, f, [8])
    assert np.allclose(a, b) and np.allclose((a ** 2).mean(-1), 1.0)


def test_weights_of_a_row_sum_to_one():
    rng = np.random.default_rng(1)
    m = small_cache(rng, [13, 7])
    q = rng.normal(size=(2, 3, 4, 8))
    for causal in (True, False):
        _, lse, _, _ = m.attention(q, causal=causal)
        score = np.full((2, 32), 2.0)
        do.weights(m, q, lse, score, causal=causal, decay=0.5)
        # 3 rows of 4 heads give a weight of 1 each, the old scores count half
        assert np.isclose(score[0, :13].sum(), 12 + 13) and np.all(score[0, 13:] == 2.0)
        do.weights(m, q, lse, score, causal=causal, decay=0.0)
        assert np.isclose(score[1, :7].sum(), 12) and np.all(score[1, 7:] == 0.0)


def test_weights_of_one_head_by_hand():
    rng = np.random.default_rng(2)
    m = small_cache(rng, [5], H=1)
    q = rng.normal(size=(1, 1, 1, 8))
    _, lse, _, _ = m.attention(q)
    score = np.zeros((1, 32))
    do.weights(m, q, lse, score)
    k = np.array([m.k[0, m.table[0][j // 4], 0, j % 4] * m.k_scale[0, m.table[0][j // 4], 0] for j in range(5)])
    x = k @ q[0, 0, 0] / math.sqrt(8)
    assert np.allclose(score[0, :5], np.exp(x) / np.exp(x).sum())


def test_evict_keeps_order_and_contents():
    rng = np.random.default_rng(3)
    m = small_cache(rng, [14, 3], n_layers=2)
    rows = [(m.k[:, m.table[0][j // 4], :, j % 4] * m.k_scale[:, m.table[0][j // 4]][..., None]).copy() for j in range(14)]
    score = np.zeros((2, 32))
    score[0, :14] = [9, 0, 5, 5, 1, math.nan, 5, 2, 8, 0, 0, 0, 7, 0]
    evicted, kept = do.evict(m, score, 7, 1, 1)
    # 0 and 13 stay; of the rest 8, 12 and the first of the fives
    assert evicted == [7, 0] and kept[0] == [0, 2, 3, 6, 8, 12, 13] and kept[1] == [-1] * 7
    assert m.len == [7, 3] and score[0, :8].tolist() == [9, 5, 5, 5, 8, 7, 0, 0]
    for i, j in enumerate(kept[0]):
        p = m.table[0][i // 4]
        got = m.k[:, p, :, i % 4] * m.k_scale[:, p][..., None]
        assert np.allclose(got, rows[j], atol=np.abs(rows[j]).max() / 8)
    assert sum(m.ref) == 2 + 1 and m.table[0][2:4] == [-1, -1]


def test_evict_leaves_the_pages_before_the_first_loss():
    rng = np.random.default_rng(4)
    m = small_cache(rng, [16])
    table = list(m.table[0])
    score = np.arange(32.0)[None].copy()
    score[0, 16:] = 0
    do.evict(m, score, 14, 9, 2)  # tokens 9 and 10 go
    assert m.table[0][:2] == table[:2] and m.table[0][2] not in table and m.len == [14]
    m = small_cache(rng, [16])
    table = list(m.table[0])
    do.evict(m, -np.arange(32.0)[None], 6)  # the tail goes: nothing moves
    assert m.table[0][:2] == table[:2] and m.table[0][2:4] == [-1, -1] and m.len == [6]


def test_evict_short_of_pages_and_given_up_pages_are_not_taken():
    rng = np.random.default_rng(5)
    m = small_cache(rng, [12, 12, 12], spare=2)
    score = rng.random((3, 32))
    score[:, :3] = -1.0
    evicted, _ = do.evict(m, score, 4)
    assert evicted == [8, 8, 0] and m.len == [4, 4, 12]
    assert do.evict(m, score, 4)[0] == [0, 0, 8]


def test_reorder_is_a_gather_of_sequences():
    rng = np.random.default_rng(6)
    m = small_cache(rng, [5, 9, 2, 12, 7, 1])
    table, length = [list(r) for r in m.table], list(m.len)
    score = rng.random((6, 32)) * (np.arange(32) < np.array(length)[:, None])
    was = score.copy()
    do.reorder(m, [[1, 1, 0], [2, 0, 5]], score=score)
    src = [1, 1, 0, 5, 3, 5]
    for s in range(6):
        n = -(-length[src[s]] // 4)
        assert m.len[s] == length[src[s]] and m.table[s][:n] == table[src[s]][:n]
        assert np.array_equal(score[s], was[src[s]])
    for p in range(m.n_pages):
        assert m.ref[p] == sum(row.count(p) for row in m.table)


def test_beam_select_brute_force():
    rng = np.random.default_rng(7)
    x = np.round(rng.normal(size=(3, 2, 9)), 1)  # (ties)
    x[:, :, 4] = -math.inf
    s = np.array([[-1.0, -1.0], [-3.0, -math.inf], [0.0, math.nan]])
    got, parent, token = do.beam_select(x, s, None, 12, 0)
    for b in range(3):
        every = []
        for w in range(2):
            for v in range(9):
                p = s[b, w] + x[b, w, v] - np.log(np.exp(x[b, w]).sum())
                every.append((-p if np.isfinite(p) else math.inf, w, v))
        every.sort(key=lambda f: (round(f[0], 9), f[1], f[2]))
        assert [f[1:] for f in every[:12]] == list(zip(parent[b], token[b]))
        assert np.allclose([f[0] for f in every[:12]], -got[b])


def test_beam_select_finished_beams():
    x = np.zeros((1, 2, 3))
    got, parent, token = do.beam_select(x, np.array([[-1.0, -2.0]]), np.array([[1, 1]]), 4, 2)
    assert parent.tolist() == [[0, 1, -1, -1]] and token.tolist() == [[2, 2, -1, -1]]
    assert got.tolist() == [[-1.0, -2.0, -math.inf, -math.inf]]
