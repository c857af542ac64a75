"""Roundings of the rotary positions, counted one by one."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2609_37581_amd import trevs
from test_gpu_cache import dev, host, storage

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("far", [4096, 1 << 20, 1 << 30])
def test_rope_rounds_each_term_once(inter, far):
    """fp32: sine and cosine (with the factor) rounded once, the products and their sum once each."""
    B, S, H, d = 2, 700, 2, 128
    rng = np.random.default_rng(far)
    x, xs = storage(rng.normal(size=(B, S, H, d)), torch.float32)
    pos = rng.integers(0, far, (1, B, S))
    freqs = co.rope_frequencies(d)
    factor = float(np.float32(1.2))
    out, _ = trevs.rope(x, None, dev(pos, torch.int64), freqs=dev(freqs, torch.float64), interleaved=inter,
                        attn_factor=factor)
    torch.cuda.synchronize()
    want = co.rope(xs, pos, freqs, [d // 2], inter, attn_factor=factor)
    first = np.arange(d // 2) * (2 if inter else 1)
    second = first + (1 if inter else d // 2)
    # |a cos w| + |b sin w| of each value, from the oracle's rotations of (a, 0) and (0, b)
    a, b = np.zeros_like(xs), np.zeros_like(xs)
    a[..., first], b[..., second] = xs[..., first], xs[..., second]
    size = sum(np.abs(co.rope(t, pos, freqs, [d // 2], inter, attn_factor=factor)) for t in (a, b))
    # a term: its cosine or sine and its product, 2^-24 each; the sum once more.  The oracle rounds pos * f in
    # 64 bits: 2^-53 of up to far / 2 pi turns, an angle off by that times 2 pi against the other term's size;
    # its own 64-bit roundings are some 2^-50
    pair = np.zeros_like(xs)
    pair[..., first] = pair[..., second] = factor * (np.abs(xs[..., first]) + np.abs(xs[..., second]))
    tol = size * 2 * 2.0 ** -24 + np.abs(want) * 2.0 ** -24
    tol = tol * (1 + 2.0 ** -20) + pair * (2 * math.pi * far * freqs.max() * 2.0 ** -53 + 2.0 ** -50)
    err = np.abs(host(out) - want)
    assert np.all(err <= tol), (err / tol).max()
