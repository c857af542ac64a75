"""The serving cache's CPU oracle against independent routines and hand
examples: torch's e4m3 conversion, masked softmax attention, complex
rotations, and the page table's invariants."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co


def test_e4m3_matches_the_format():
    table = co.e4m3_bytes()
    nums = np.sort(table[np.isfinite(table)])
    assert nums.max() == 448.0 and np.abs(nums[nums != 0]).min() == 2.0 ** -9
    assert np.array_equal(co.e4m3(nums), nums)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=2000) * 100, rng.normal(size=2000) * 0.01, (nums[1:] + nums[:-1]) / 2])
    x = x[np.abs(x) <= 448].astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(co.e4m3(x), want)


def test_block_scale_is_the_smallest():
    x = np.array([0.0, 448.0, np.nextafter(448.0, 500), 1.0, 1.75, 1.76, 3e38, 1e-45, 448 * 2.0 ** -126])
    s = co.block_scale(x)
    assert np.all(np.log2(s) == np.rint(np.log2(s))) and np.all(x <= 448 * s)
    assert s.tolist() == [2.0 ** -126, 1.0, 2.0, 2.0 ** -8, 2.0 ** -8, 2.0 ** -7, 2.0 ** 120, 2.0 ** -126, 2.0 ** -126]


@pytest.mark.parametrize("inter", [False, True])
def test_rope_is_a_complex_rotation(inter):
    rng = np.random.default_rng(1)
    x, pos = rng.normal(size=(2, 3, 4, 64)), rng.integers(0, 9, (2, 2, 3))
    f = co.rope_frequencies(32, base=100.0)
    y = co.rope(x, pos, f, [5, 11], inter, attn_factor=1.5)
    a, b = (slice(0, 32, 2), slice(1, 32, 2)) if inter else (slice(0, 16), slice(16, 32))
    z = x[..., a] + 1j * x[..., b]
    p = np.concatenate([np.repeat(pos[0][..., None], 5, -1), np.repeat(pos[1][..., None], 11, -1)], -1)
    w = z * np.exp(2j * math.pi * p * f)[:, :, None] * 1.5
    assert np.allclose(y[..., a], w.real, atol=1e-12) and np.allclose(y[..., b], w.imag, atol=1e-12)
    assert np.array_equal(y[..., 32:], x[..., 32:])
    back = co.rope(y / 1.5, pos, f, [5, 11], inter, inverse=True)
    assert np.allclose(back[..., :32], x[..., :32], atol=1e-12)


def test_attention_matches_torch():
    rng = np.random.default_rng(2)
    m = co.CacheModel(n_pages=12, page=16, n_slots=2, max_pages=5, H_kv=2, d=64)
    m.reserve([37, 5])
    k, v = rng.normal(size=(2, 2, 40, 2, 64))
    m.write(k[:, :37], v[:, :37], [37, 5])
    q = rng.normal(size=(2, 3, 4, 64))
    out, lse, _, _ = m.attention(q, q_len=[3, 2])
    ids = m.table[0][:3]
    K = torch.from_numpy(np.concatenate([m.k[0, p] * m.k_scale[0, p][:, None, None] for p in ids], 1)[:, :37])
    V = torch.from_numpy(np.concatenate([m.v[0, p] * m.v_scale[0, p][:, None, None] for p in ids], 1)[:, :37])
    Q = torch.from_numpy(q[0]).transpose(0, 1)
    mask = torch.ones(3, 37, dtype=torch.bool).tril(34)
    want = torch.nn.functional.scaled_dot_product_attention(Q, K.repeat_interleave(2, 0), V.repeat_interleave(2, 0),
                                                            attn_mask=mask).transpose(0, 1)
    assert np.allclose(out[0], want.numpy(), atol=1e-12)
    assert np.isnan(out[1, 2]).all() and np.isfinite(out[1, :2]).all()


def test_write_keeps_values_within_half_a_step():
    """A value's error is at most half an e4m3 step of the largest scale its
    block had, plus a quarter for every time that scale rose (subnormals)."""
    rng = np.random.default_rng(3)
    m = co.CacheModel(n_pages=3, page=16, n_slots=1, max_pages=2, H_kv=1, d=64)
    rows = []
    for t in range(20):
        m.reserve([1])
        x = rng.normal(size=(1, 1, 1, 64)) * 2.0 ** (t % 7)
        rows.append(x[0, 0, 0])
        m.write(x, -x)
    for t, x in enumerate(rows):
        p = m.table[0][t // 16]
        s = m.k_scale[0, p, 0]
        got = m.k[0, p, 0, t % 16] * s
        assert np.all(np.abs(got - x) <= np.abs(x) * 2.0 ** -4 + 4 * s * 2.0 ** -10)
        assert np.array_equal(m.v[0, p, 0, t % 16], -m.k[0, p, 0, t % 16])


def test_page_table_invariants():
    rng = np.random.default_rng(4)
    m = co.CacheModel(n_pages=24, page=16, n_slots=8, max_pages=6, H_kv=1, d=64)
    for _ in range(300):
        op = rng.integers(3)
        slots = rng.integers(-1, 9, 3).tolist()
        if op == 0:
            m.reserve(rng.integers(0, 40, 3).tolist(), slots)
        elif op == 1:
            m.fork(rng.integers(-1, 9, 3).tolist(), slots, rng.integers(0, 90, 3).tolist())
        else:
            m.free(slots, rng.integers(0, 50, 3).tolist() if rng.random() < 0.5 else None)
        held = [0] * 24
        for s in range(8):
            n = -(-m.len[s] // 16)
            assert all(p >= 0 for p in m.table[s][:n]) and all(p == -1 for p in m.table[s][n:])
            for p in m.table[s][:n]:
                held[p] += 1
        assert held == m.ref


def test_fork_then_append_copies_the_shared_page_once():
    m = co.CacheModel(n_pages=8, page=16, n_slots=3, max_pages=4, H_kv=1, d=64)
    m.reserve([20])
    assert m.fork([0, 0], [1, 2]) == [1, 1]
    assert m.ref[:2] == [3, 3]
    granted, src, dst = m.reserve([1, 1, 1])
    # the first two take copies of page 1, the last holder keeps it
    assert granted == [1, 1, 1] and src == [1, 1, -1] and dst == [2, 3, -1]
    assert m.ref[:4] == [3, 1, 1, 1] and m.table[2][:2] == [0, 1]
