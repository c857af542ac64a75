"""The decode loop on the GPU against its float64 oracle: head norms with the
rotation, attention weights summed for each cached token, eviction by them, beam
search's selection, the beams' sequences reordered, and a run of them together."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from oracle import decode_oracle as do
from paper_2609_37581_amd import trevs
from test_gpu_cache import check_contents, check_table, dev, device_cache, host, model, storage

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]


# ---------------------------------------------------------------- head norms
NORM = [  # B, S, H_q, H_k, d, rot, sections, far, per_head, offset
    (1, 1, 1, 0, 64, 16, [8], 100, False, 0.0), (2, 3, 7, 1, 128, 128, [16, 24, 24], 4096, False, 1.0),
    (3, 37, 4, 4, 64, 48, [0, 24], 70000, True, 0.0), (1, 300, 28, 4, 128, 64, [32], 1 << 20, True, 1.0),
    (2, 5, 3, 2, 256, 256, [128], 1 << 33, False, 0.0), (5, 1, 32, 8, 128, 128, [1, 2, 60, 1], 999, True, -0.5),
    (1, 1100, 2, 2, 256, 16, [8], 32768, False, 1.0),
]


def check_norm(got, x, w, offset, eps, pos, f, sections, inter, gain, dtype):
    d, half = x.shape[-1], len(f)
    want, y = do.norm_rope(x, w, offset, eps, pos, f, sections, inter, gain)
    # the sum of squares is off by d roundings and halves under the root, then a root, a weight's sum and two
    # products; the turn as without the norm: the angle by 2 pi 2^-25 (its fraction cast to 32 bits), sine, cosine,
    # their factor, two products and a sum by 2^-24 each and two ulps for the functions
    rel = ((d + 4) / 2 + 8) * 2.0 ** -24
    first = np.arange(half) * (2 if inter else 1)
    second = first + (1 if inter else half)
    # (a weight near -offset loses relative precision in its sum)
    z = np.abs(y) if w is None else np.abs(x) / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * (np.abs(w) + abs(offset))
    tol = z * rel
    pair = gain * (z[..., first] + z[..., second])
    turns = 2 * math.pi * (2.0 ** -25 + np.abs(pos).max() * np.abs(f).max() * 2.0 ** -53) + 8 * 2.0 ** -24
    tol[..., first] = tol[..., second] = pair * (rel + turns)
    tol = tol + (np.abs(want) + tol) * torch.finfo(dtype).eps / 2
    err = np.abs(host(got) - want)
    assert np.all(err <= tol), (err / tol).max()


@pytest.mark.parametrize("shape", NORM)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("inter", [False, True])
def test_norm_rope(shape, dtype, inter):
    B, S, H_q, H_k, d, rot, sections, far, per_head, offset = shape
    print(f"[norm] {shape} {dtype} {inter}", flush=True)
    rng = np.random.default_rng(B * 7 + S)
    pos = rng.integers(0, far, (len(sections), B, S))
    f = co.rope_frequencies(rot, base=500.0)
    fd, pd = dev(f, torch.float64), dev(pos, torch.int64)
    # q and k as slices of a fused projection with values behind them
    H = H_q + 2 * H_k
    fused, x = storage(rng.normal(size=(B, S, H, d)) * np.exp2(rng.integers(-3, 4, (B, S, H, 1))), dtype)
    q, k = fused[:, :, :H_q], fused[:, :, H_q:H_q + H_k] if H_k else None
    before = fused.clone()
    for wt in DTYPES:
        wq, vq = storage(rng.normal(size=(H_q, d) if per_head else (d,)) + 1 - offset, wt)
        wk, vk = storage(rng.normal(size=(H_k, d) if per_head else (d,)) + 1 - offset, wt) if H_k else (None, None)
        if wt == torch.float32 and S == 3:
            wq, vq = None, None  # (one tensor without weights)
        kw = dict(freqs=fd, q_weight=wq, k_weight=wk, eps=1e-5, weight_offset=offset, sections=sections,
                  interleaved=inter, attn_factor=1.25)
        call = trevs.NormRope(q, k, pd, **kw)
        call()
        torch.cuda.synchronize()
        assert torch.equal(fused, before)
        eps = float(np.float32(1e-5))
        check_norm(call.q_out, x[:, :, :H_q], vq, offset, eps, pos, f, sections, inter, 1.25, dtype)
        if H_k:
            check_norm(call.k_out, x[:, :, H_q:H_q + H_k], vk, offset, eps, pos, f, sections, inter, 1.25, dtype)
        # in place, the same bits, and nothing else of the buffer changes
        trevs.norm_rope(q, k, pd, inplace=True, **kw)
        torch.cuda.synchronize()
        assert torch.equal(q, call.q_out) and (not H_k or torch.equal(k, call.k_out))
        assert torch.equal(fused[:, :, H_q + H_k:], before[:, :, H_q + H_k:])
        fused.copy_(before)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_norm_rope_magnitudes(dtype, d):
    """Rows whose squares leave fp32's range, up and down, beside ordinary and zero ones."""
    rng = np.random.default_rng(d)
    x = rng.normal(size=(1, 6, 2, d)).clip(-3, 3)
    x *= np.array([1.0, 2.0 ** 125, 2.0 ** 66, 2.0 ** -100, 2.0 ** -45, 0.0])[None, :, None, None]
    x[0, 1, 1], x[0, 3, 1] = 0.0, 0.0
    x[0, 1, 1, d // 2], x[0, 3, 1, d // 2] = 3.3e38, 2.0 ** -120  # one value alone
    q, xs = storage(x, dtype)
    pos, f = np.arange(6)[None, None], co.rope_frequencies(d)
    for eps in (1e-6, 1e-12, 2.0 ** -126):
        got, none = trevs.norm_rope(q, None, dev(pos, torch.int64), freqs=dev(f, torch.float64), eps=eps)
        assert none is None and torch.isfinite(got.float()).all()
        check_norm(got, xs, None, 0.0, float(np.float32(eps)), pos, f, [d // 2], False, 1.0, dtype)
        assert (got[0, 5] == 0).all()


def test_norm_rope_offsets_past_32_bits():
    """The last rows of 4.6 GB, in place, give the bits that they give alone."""
    S, H, d = 140000, 32, 256
    q = torch.zeros(1, S, H, d, device="cuda")
    rows, _ = storage(np.random.default_rng(3).normal(size=(1, 7, H, d)), torch.float32)
    q[:, -7:] = rows
    pos = torch.arange(S, device="cuda")[None, None]
    kw = dict(freqs=dev(co.rope_frequencies(64), torch.float64), q_weight=torch.rand(H, d, device="cuda"))
    want, _ = trevs.norm_rope(rows, None, pos[:, :, -7:].contiguous(), **kw)
    trevs.norm_rope(q, None, pos, inplace=True, **kw)
    assert torch.equal(q[:, -7:], want) and not q[:, :-7].any()


# ------------------------------------------------------------ summed weights
def scores_for(m, c, rng):
    s = trevs.kv8_scores(c)
    x = rng.random(tuple(s.shape)) * (np.arange(s.shape[1]) < np.clip(np.array(m.len)[:, None], 0, None))
    s.copy_(torch.from_numpy(x).float())
    return s, host(s)


def check_weights(got, want, total, spread, count, decay, old):
    # a weight's exponent is off by 2^-24 of what enters its logit, its log-sum-exp and their difference, its
    # exponential by 2^-22; fp32 sums of `count` of them, a product with the decay and a sum
    tol = np.expm1(spread * 2.0 ** -24 / np.maximum(total, 1e-300)) * total + 2.0 ** -22 * total
    tol = tol + (count + 4) * 2.0 ** -24 * (total + tol) + 2.0 ** -23 * (decay * np.abs(old) + np.abs(want))
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    err = np.abs(got - want)
    assert np.all((err <= tol + 1e-37)[~nan]), (np.nanmax(np.where(nan, 0, err / (tol + 1e-37))), np.nanmax(err))


def run_weights(m, c, q, qs, rng, q_len=None, slots=None, kv_max=0, decay=1.0, causal=True, scale=None, layer=0, lse=None):
    if lse is None:
        _, lse, _, _ = m.attention(qs, q_len=q_len, slots=slots, kv_max=kv_max, causal=causal, scale=scale, layer=layer)
    ld, lse = storage(np.where(np.isnan(lse), 9e9, lse), torch.float32)  # (rows past q_len: not read)
    score, want = scores_for(m, c, rng)
    old = want.copy()
    kw = dict(kv_max=kv_max, causal=causal, scale=scale, layer=layer)
    decay = float(np.float32(decay))
    bound = do.weights(m, qs, lse, want, q_len=q_len, slots=slots, decay=decay, **kw)
    call = trevs.Kv8Weights(c, q, ld, score, None if q_len is None else dev(q_len), None if slots is None else dev(slots),
                            decay=decay, **kw)
    assert call() is score
    check_weights(host(score), want, *bound, decay, old)
    first = score.clone()
    score.copy_(torch.from_numpy(old))
    call()
    assert torch.equal(first.view(torch.int32), score.view(torch.int32))  # the same bits again
    return score


WEIGHTS = [  # page, H_q, H_kv, d, T, lens
    (16, 4, 4, 64, 1, [1, 16, 17, 0, 333]), (64, 7, 1, 128, 1, [64, 63, 65, 1, 1000]),
    (32, 28, 4, 128, 1, [700, 31, 32]), (16, 40, 2, 128, 1, [100, 257]), (64, 8, 1, 256, 1, [129, 5]),
    (32, 6, 2, 64, 5, [3, 40, 0, 5]), (16, 28, 4, 128, 3, [200, 3, 19]), (64, 28, 4, 128, 33, [64, 33, 500]),
    (32, 4, 4, 128, 70, [70, 200, 129]), (64, 2, 2, 256, 45, [45, 300]), (16, 3, 1, 64, 130, [131, 100]),
    (64, 16, 2, 64, 17, [400]), (32, 8, 1, 256, 40, [90]), (16, 33, 1, 64, 1, [77, 15]), (64, 1, 1, 128, 150, [150]),
    (16, 20, 20, 64, 2, [50, 300, 2]), (32, 32, 1, 128, 1, [65]), (64, 5, 5, 64, 270, [270, 600]),
]


@pytest.mark.parametrize("shape", WEIGHTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_weights(shape, dtype, causal):
    page, H_q, H_kv, d, T, lens = shape
    print(f"[weights] {shape} {dtype} {causal}", flush=True)
    rng = np.random.default_rng(sum(lens) + d)
    m = model(rng, lens, page, H_kv, d)
    c = device_cache(m)
    fused, x = storage(rng.normal(size=(len(lens), T, H_q + 3, d)), dtype)
    q, qs = fused[:, :, :H_q], x[:, :, :H_q]
    q_len = [max(0, T - 2 * b) for b in range(len(lens))]
    run_weights(m, c, q, qs, rng, q_len=q_len, causal=causal, decay=0.75)
    run_weights(m, c, q, qs, rng, causal=causal, kv_max=max(lens), scale=0.31, decay=0.0)


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("dtype", DTYPES)
def test_weights_masked_places_hold_anything(T, dtype):
    """NaN bytes behind the last token, in pages of no sequence and in unused
    scales, NaN in scores that are begun anew and behind the rows; absent pages;
    lengths past the table; a slot out of range; lengths cut by kv_max."""
    print(f"[weights masked] {T} {dtype}", flush=True)
    rng = np.random.default_rng(5)
    m = model(rng, [150, 37, 260, 64, 90], 32, 2, 128, spare=6)
    m.table[0][1] = -5
    m.table[2][0], m.table[2][8] = m.n_pages + 3, -1
    m.table[3] = [-1] * m.max_pages
    c = device_cache(m)
    used = set()
    for s in range(5):
        for j in range(-(-m.len[s] // 32)):
            p, n = m.table[s][j], min(32, m.len[s] - 32 * j)
            if 0 <= p < m.n_pages:
                used.add(p)
                c.k[0, p, :, n:] = 0x7f
    for p in set(range(m.n_pages)) - used:
        c.k[0, p], c.k_scale[0, p] = 0xff, math.nan
    q, qs = storage(rng.normal(size=(5, T, 4, 128)), dtype)
    for causal in (True, False):
        run_weights(m, c, q, qs, rng, causal=causal, decay=0.5)
        run_weights(m, c, q, qs, rng, causal=causal, slots=[4, 2, 0, 3, 99], kv_max=100)
    # scores begun anew do not look at what was there, those that are not keep it
    _, lse, _, _ = m.attention(qs)
    ld, lse = storage(lse, torch.float32)
    for decay in (0.0, 1.0):
        score = trevs.kv8_scores(c).fill_(math.nan)
        want = np.zeros(tuple(score.shape))
        bound = do.weights(m, qs, lse, want, decay=0.0)
        trevs.kv8_weights(c, q, ld, score, decay=decay)
        if decay:
            assert torch.isnan(score).all()
        else:
            check_weights(host(score), want, *bound, 0.0, 0 * want)


@pytest.mark.parametrize("T", [1, 3, 50])
@pytest.mark.parametrize("dtype", DTYPES)
def test_weights_nan_keys_and_rows(T, dtype):
    """A NaN key reaches its own token's score, a row's NaN log-sum-exp what the row sees, and
    rows whose log-sum-exp is -inf give nothing."""
    rng = np.random.default_rng(T)
    m = model(rng, [90, 70], 16, 1, 64)
    m.k[0, m.table[0][2], 0, 5, 7] = 0.0
    c = device_cache(m)
    q, qs = storage(rng.normal(size=(2, T, 4, 64)), dtype)
    _, lse, _, _ = m.attention(qs)
    c.k[0, m.table[0][2], 0, 5, 7] = 0x7f
    m.k[0, m.table[0][2], 0, 5, 7] = math.nan
    lse[0, 1, 0] = -math.inf
    lse[1, 2, T // 2] = math.nan
    lse[1, 3, :] = -math.inf
    ld, ls = storage(lse, torch.float32)
    score, want = scores_for(m, c, rng)
    old = want.copy()
    bound = do.weights(m, qs, ls, want)
    trevs.kv8_weights(c, q, ld, score)
    assert np.isnan(want[0, 37]) and np.isnan(want[0]).sum() == 1
    bound = [np.nan_to_num(b) for b in bound]
    check_weights(host(score), want, *bound, 1.0, old)


@pytest.mark.parametrize("T", [1, 60])
@pytest.mark.parametrize("dtype", DTYPES)
def test_weights_large_logits_and_far_scales(T, dtype):
    rng = np.random.default_rng(6)
    m = model(rng, [300, 65], 16, 2, 64)
    m.k_scale *= np.exp2(rng.integers(-30, 6, m.k_scale.shape))
    m.k[0, m.table[0][3]], m.k_scale[0, m.table[0][3]] = 0.0, 2.0 ** -126
    c = device_cache(m)
    q, qs = storage(rng.normal(size=(2, T, 4, 64)) * 4, dtype)
    run_weights(m, c, q, qs, rng)
    run_weights(m, c, q, qs, rng, scale=1e-12, decay=2.5)


@pytest.mark.parametrize("T,H_q,H_kv", [(1, 2, 1), (2, 40, 2), (9, 8, 2), (40, 8, 2)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_weights_of_many_uneven_sequences_without_a_bound(T, H_q, H_kv, dtype):
    print(f"[weights uneven] {T} {H_q} {H_kv} {dtype}", flush=True)
    rng = np.random.default_rng(T)
    B = 70
    lens = [int(n) for n in rng.integers(0, 90, B)]
    for i in (0, 5, 63, 64, 65, B - 1):
        lens[i] = int(rng.integers(200, 400))
    lens[7] = 0
    m = model(rng, lens, 16, H_kv, 64)
    m.max_pages = 256
    m.table = [row + [-1] * (256 - len(row)) for row in m.table]
    c = device_cache(m)
    q, qs = storage(rng.normal(size=(B, T, H_q, 64)), dtype)
    q_len = rng.integers(0, T + 1, B).tolist()
    run_weights(m, c, q, qs, rng, q_len=q_len, decay=0.0)
    run_weights(m, c, q, qs, rng, q_len=[0] * B, decay=0.5)  # no work at all
    run_weights(m, c, q, qs, rng, q_len=[0] * B, decay=0.0)


def test_weights_under_a_very_long_table():
    """So long that heads share their parts of the workspace, and that a launch does not
    have a workgroup for each of its blocks of zeros."""
    rng = np.random.default_rng(8)
    for T in (1, 40):
        m = model(rng, [500, 77, 0], 16, 4, 64)
        m.max_pages = 400000
        m.table = [row + [-1] * (m.max_pages - len(row)) for row in m.table]
        c = device_cache(m)
        q, qs = storage(rng.normal(size=(3, T, 8, 64)), torch.bfloat16)
        run_weights(m, c, q, qs, rng, decay=0.0)
        run_weights(m, c, q, qs, rng, kv_max=600, decay=0.0)


def test_weights_second_layer_and_offsets_past_32_bits():
    page, H, d, n_pages = 64, 32, 256, 8300  # 4.3 GB a layer and side
    c = trevs.Kv8Cache(n_pages=n_pages, page_tokens=page, n_slots=2, max_pages=3, H_kv=H, d_head=d)
    top = n_pages - 1
    m = co.CacheModel(10, page, 2, 3, H, d)
    m.table, m.len, m.ref = [[9, 0, 8], [7, 6, -1]], [150, 100], [1, 0, 0, 0, 0, 0, 1, 1, 1, 1]
    far = lambda p: p if p < 6 else top - (9 - p)  # noqa: E731  model page -> device page
    c.table.copy_(dev([[far(p) if p >= 0 else -1 for p in row] for row in m.table]))
    c.len.copy_(dev(m.len))
    for p in (0, 6, 7, 8, 9):
        c.ref[far(p)] = 1
    rng = np.random.default_rng(8)
    k, ks = storage(rng.normal(size=(2, 150, H, d)), torch.bfloat16)
    trevs.kv8_write(c, k, -k, dev([150, 100]))
    m.write(ks, -ks, [150, 100])
    for T in (1, 40):
        q, qs = storage(rng.normal(size=(2, T, H, d)), torch.bfloat16)
        run_weights(m, c, q, qs, rng)
    # and evicted from there
    score, want = scores_for(m, c, rng)
    got = trevs.kv8_evict(c, score, n_keep=70, n_first=3)
    assert [t.tolist() for t in got] == [list(x) for x in do.evict(m, want, 70, 3)]
    torch.cuda.synchronize()
    table = {}
    for s in range(2):
        for a, b in zip(c.table[s].tolist(), m.table[s]):
            assert (a < 0) == (b < 0)
            table[b] = a
    TABLE = co.e4m3_bytes()
    for b, a in table.items():
        if b >= 0:
            assert np.array_equal(TABLE[c.k[0, a].cpu().numpy()], m.k[0, b])
            assert np.array_equal(TABLE[c.v[0, a].cpu().numpy()].swapaxes(1, 2), m.v[0, b])
    m = model(rng, [60, 33], 16, 2, 64, n_layers=2)
    c = device_cache(m)
    q, qs = storage(rng.normal(size=(2, 2, 4, 64)), torch.float32)
    run_weights(m, c, q, qs, rng, layer=1)


# ------------------------------------------------------------------ eviction
def run_evict(m, c, score, want, slots=None, keep=None, **kw):
    got = trevs.kv8_evict(c, score, None if slots is None else dev(slots), keep=None if keep is None else dev(keep), **kw)
    lists = do.evict(m, want, slots=slots, keep=keep, **kw)
    assert [t.tolist() for t in got] == [list(x) for x in lists]
    check_table(c, m)
    for s in range(m.n_slots):  # (entries behind a sequence are not read, but eviction leaves -1)
        n = -(-min(max(m.len[s], 0), m.max_pages * m.page) // m.page)
        if any(e > 0 and (s if slots is None else slots[i]) == s for i, e in enumerate(lists[0])):
            assert c.table[s].tolist()[n:] == m.table[s][n:], s
    assert np.array_equal(host(score), want, equal_nan=True)
    check_contents(c, m)
    return lists


@pytest.mark.parametrize("page,H,d", [(16, 2, 64), (32, 1, 256), (64, 3, 128)])
def test_evict(page, H, d):
    print(f"[evict] {page} {H} {d}", flush=True)
    rng = np.random.default_rng(page)
    lens = [3 * page + 5, 70, 69, 71, 1, 0, 8 * page, 5 * page - 1, 200]
    m = model(rng, lens, page, H, d, n_layers=2, spare=30)
    m.table[8][1] = -1  # rows of a page that is not there are zeros
    c = device_cache(m)
    score, want = scores_for(m, c, rng)
    score[6, ::3], want[6, ::3] = 0.5, 0.5      # ties
    score[7, 4:90:5], want[7, 4:90:5] = math.nan, math.nan
    score[7, 3], want[7, 3] = math.inf, math.inf
    score[7, 6], want[7, 6] = -math.inf, -math.inf
    score[7, 8], score[7, 9], want[7, 8:10] = -0.0, 0.0, 0.0
    run_evict(m, c, score, want, n_keep=70, n_first=2, n_last=10)
    # some of them further, with budgets of their own, in another order; one slot twice, others out of range
    run_evict(m, c, score, want, slots=[7, 3, 99, 0, 7, 6, -1, 8], keep=[33, 64, 5, -4, 20, 1000, 3, page],
              n_keep=65, n_first=0, n_last=1)
    run_evict(m, c, score, want, n_keep=1)


@pytest.mark.parametrize("case", ["tail", "head", "all held", "one", "page", "same page"])
def test_evict_extremes(case):
    """Nothing moves; everything does; no choice at all; one token is kept; whole pages
    are; only the last page changes."""
    rng = np.random.default_rng(9)
    for page in (16, 64):
        L = 5 * page + 3
        m = model(rng, [L, L], page, 1, 64, spare=12)
        c = device_cache(m)
        score, want = scores_for(m, c, rng)
        order = np.arange(want.shape[1], dtype=float)
        order = {"tail": -order, "head": order, "same page": -order}.get(case, rng.permutation(order))
        want[:] = np.where(np.arange(want.shape[1]) < L, order, 0.0)
        score.copy_(torch.from_numpy(want))
        kw = {"tail": dict(n_keep=2 * page + 7), "head": dict(n_keep=2 * page), "all held": dict(n_keep=50, n_first=20, n_last=30),
              "one": dict(n_keep=1), "page": dict(n_keep=3 * page, n_first=page), "same page": dict(n_keep=L - 1, n_last=2)}[case]
        run_evict(m, c, score, want, **kw)


def test_evict_shared_pages_and_shortage():
    """Forks of one image: pages before the first loss stay shared, the others are read and given
    up; requests that the free pages do not cover are passed over, smaller ones behind them served."""
    for spare in (0, 1, 3, 7, 40):
        rng = np.random.default_rng(spare)
        m = model(rng, [200, 90], 16, 1, 64, spare=spare, slots=None)
        m.n_slots = 6
        m.table += [[-1] * m.max_pages for _ in range(4)]
        m.len += [0] * 4
        m.fork([0, 0, 1, 0], [2, 3, 4, 5], [200, 150, 90, 200])
        c = device_cache(m)
        score, want = scores_for(m, c, rng)
        want[:, :40] += 5.0
        want *= np.arange(want.shape[1]) < np.array(m.len)[:, None]
        want = want.astype(np.float32).astype(float)
        score.copy_(torch.from_numpy(want))
        lists = run_evict(m, c, score, want, slots=[2, 0, 3, 4], keep=[120, 60, 41, 17], n_keep=128, n_first=4, n_last=8)
        run_evict(m, c, score, want, n_keep=64, n_first=32)
        assert spare or lists[0][:3] == [0, 0, 0]


@pytest.mark.parametrize("L", [1025, 5000, 17000, 40000, 66000])
def test_evict_long_sequences(L):
    """Every size of the selection, the last one past what it holds in registers."""
    print(f"[evict long] {L}", flush=True)
    rng = np.random.default_rng(L)
    m = model(rng, [L, 100, L // 2], 64, 1, 64, spare=L // 64)
    c = device_cache(m)
    score, want = scores_for(m, c, rng)
    want[:] = np.round(want, 3)  # (ties)
    want[:] = want.astype(np.float32)
    score.copy_(torch.from_numpy(want))
    run_evict(m, c, score, want, n_keep=L // 3, n_first=5, n_last=64)


def test_evict_many_requests():
    rng = np.random.default_rng(4)
    n = trevs.MAX_PAGE_REQUESTS
    lens = rng.integers(0, 60, n).tolist()
    m = model(rng, lens, 16, 1, 64, spare=500)
    c = device_cache(m)
    score, want = scores_for(m, c, rng)
    run_evict(m, c, score, want, n_keep=20, n_first=1, n_last=2)
    run_evict(m, c, score, want, slots=rng.integers(-1, n + 1, n).tolist(), n_keep=9)


# --------------------------------------------------------------- beam search
def check_beams(got, x, s, done, n_out, eos):
    """x, s: the float64 values of the call's logits and scores."""
    score, parent, token = host(got[0]), got[1].cpu().numpy(), got[2].cpu().numpy()
    want, wp, wt = do.beam_select(x, s, done, n_out, eos)
    # log of a sum whose terms are off by 2^-22 and the rounding of an argument of up to 16 that matters, in sums
    # of 32 and then 10 terms in 32 bits; the result is rounded once
    tol = 80 * 2.0 ** -24
    same = (score == want) | (np.abs(score - want) <= tol + 2.0 ** -24 * np.abs(want))
    assert np.all(same), (score[~same], want[~same])
    for b in range(len(want)):
        pairs = list(zip(parent[b], token[b]))
        real = [p for p in pairs if p != (-1, -1)]
        assert len(set(real)) == len(real)
        for r in range(n_out):
            # only continuations of different beams can be closer together than the bound without being equal
            near = [i for i in range(n_out) if i != r and wp[b, i] != wp[b, r] and want[b, i] > -math.inf
                    and abs(want[b, i] - want[b, r]) <= 2 * tol]
            if near:
                assert pairs[r] in [(wp[b, i], wt[b, i]) for i in near + [r]]
            elif r < n_out - 1:
                assert pairs[r] == (wp[b, r], wt[b, r]), (b, r, pairs, wp[b], wt[b])


BEAMS = [  # B, W, V, n_out, pad
    (1, 1, 1, 1, 0), (2, 3, 5, 7, 0), (1, 4, 32000, 8, 0), (3, 2, 8192, 5, 3), (2, 5, 8193, 10, 1), (1, 64, 700, 64, 0),
    (2, 8, 20011, 16, 5), (1, 1, 70000, 64, 0), (5, 3, 333, 3, 2), (1, 2, 40, 64, 0), (17, 4, 8191, 4, 0),
]


@pytest.mark.parametrize("shape", BEAMS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_beam_select(shape, dtype):
    B, W, V, n, pad = shape
    print(f"[beam] {shape} {dtype}", flush=True)
    rng = np.random.default_rng(V + W)
    full, x = storage(rng.normal(size=(B, W, V + pad)) * 3, dtype)
    logits, x = full[:, :, :V], x[:, :, :V]
    score, s = storage(-10 * rng.random((B, W)), torch.float32)
    got = trevs.beam_select(logits, score, n_out=n)
    check_beams(got, x, s, None, n, 0)
    done = rng.random((B, W)) < 0.4
    eos = int(rng.integers(0, V))
    got = trevs.beam_select(logits, score, dev(done), n_out=n, eos=eos)
    check_beams(got, x, s, done, n, eos)


@pytest.mark.parametrize("dtype", DTYPES)
def test_beam_select_ties_and_banned_tokens(dtype):
    """All logits equal; nearly all banned; few values; equal beams; sorted logits; beams that are
    not in use; NaN and infinities: more candidates than the lists hold, and rows without any."""
    rng = np.random.default_rng(3)
    V, n = 20000, 12
    x = np.zeros((10, 3, V))
    x[1] = -math.inf
    x[1, :, 17000:17005] = rng.normal(size=(3, 5))
    x[2] = np.round(rng.normal(size=(3, V)))
    x[3] = np.round(rng.normal(size=V) * 4)  # three equal beams
    x[4] = np.arange(V) / 64.0
    x[5] = -np.arange(V) / 64.0
    x[6] = rng.normal(size=(3, V))
    x[6, 0, 5], x[6, 1, 19999], x[6, 2] = math.nan, math.inf, -math.inf
    x[7] = rng.normal(size=(3, V))
    x[8] = -math.inf
    x[9, :, ::2] = -0.0
    logits, xs = storage(x, dtype)
    score, s = storage(np.tile([[-1.0, -1.5, -1.25]], (10, 1)), torch.float32)
    s[3], s[0] = -2.0, [-1.0, -1.0, -3.0]
    s[7] = [-math.inf, math.nan, math.inf]
    s[6, 0] = -0.5
    score.copy_(torch.from_numpy(s))
    got = trevs.beam_select(logits, score, n_out=n)
    check_beams(got, xs, s, None, n, 0)
    assert got[1][0].tolist() == [0] * 12 and got[2][0].tolist() == list(range(12))
    done = np.zeros((10, 3), bool)
    done[6] = done[7] = True
    got = trevs.beam_select(logits, score, dev(done), n_out=n, eos=3)
    check_beams(got, xs, s, done, n, 3)
    assert got[1][6].tolist()[3:] == [-1] * 9


def test_beam_select_does_not_depend_on_where_rows_lie():
    """Equal beams at every alignment give equal scores: they tie, and the lower beam wins."""
    rng = np.random.default_rng(12)
    for dtype in DTYPES:
        row, _ = storage(rng.normal(size=9001) * 2, dtype)
        logits = row.expand(2, 16, 9001).contiguous()
        got = trevs.beam_select(logits, torch.zeros(2, 16, device="cuda"), n_out=16)
        assert got[1].tolist() == [list(range(16))] * 2
        assert len(set(got[2].flatten().tolist())) == 1


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shift", [0.0, 7e4, -7e4, 1e9, -3e30, 2e38])
def test_beam_select_logits_far_from_zero(dtype, shift):
    """Logits up to the largest floats, beside beams of ordinary ones; chunks of either kind in one beam."""
    rng = np.random.default_rng(9)
    x = rng.normal(size=(2, 3, 9000)) * max(1.0, abs(shift) / 4) + shift
    x = x.clip(-3.3e38, 3.3e38)
    x[0, 1] = rng.normal(size=9000)
    x[1, 2, :4500] = rng.normal(size=4500)
    logits, xs = storage(x, dtype)
    score, s = storage(np.array([[-1.0, -2.0, -0.5], [-3.0, -1.0, -2.0]]), torch.float32)
    check_beams(trevs.beam_select(logits, score, n_out=9), xs, s, None, 9, 0)


def test_beam_select_more_ties_than_the_join_lists():
    """Every listed continuation of 64 beams ties."""
    score = torch.zeros(2, 64, device="cuda")
    got = trevs.beam_select(torch.zeros(2, 64, 9000, device="cuda"), score, n_out=64)
    assert got[1].tolist() == [[0] * 64] * 2 and got[2].tolist() == [list(range(64))] * 2


def test_beam_select_offsets_past_32_bits():
    """Six rows of 4e8 logits, 4.8 GB."""
    V = 400_000_000
    logits = torch.zeros(3, 2, V, dtype=torch.bfloat16, device="cuda")
    logits[2, 1, V - 1], logits[2, 1, 7], logits[2, 0, V - 5], logits[0, 1, 9], logits[0, 0, 3] = 12.0, 11.0, 10.0, 9.0, 8.0
    logits[1, 0, V // 2], logits[1, 0, 0] = 3.0, 2.0
    score = torch.tensor([[0.0, -0.5], [-1.0, -9.0], [0.0, -0.25]], device="cuda")
    got = trevs.beam_select(logits, score, n_out=2)
    sums = [[V - 1 + math.exp(8), V - 1 + math.exp(9)], [V - 2 + math.exp(3) + math.exp(2), V],
            [V - 1 + math.exp(10), V - 2 + math.exp(12) + math.exp(11)]]
    want = [[(-0.5 + 9, 1, 9), (8.0, 0, 3)], [(-1.0 + 3, 0, V // 2), (-1.0 + 2, 0, 0)], [(-0.25 + 12, 1, V - 1), (-0.25 + 11, 1, 7)]]
    assert got[1].tolist() == [[w for _, w, _ in row] for row in want]
    assert got[2].tolist() == [[v for _, _, v in row] for row in want]
    exact = np.array([[x - math.log(sums[b][w]) for x, w, _ in row] for b, row in enumerate(want)])
    assert np.all(np.abs(host(got[0]) - exact) <= 80 * 2.0 ** -24 + 2.0 ** -24 * np.abs(exact))


# ------------------------------------------------------------------- reorder
@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("groups,W", [(1, 1), (1, 4), (5, 3), (3, 64), (128, 8)])
def test_reorder(groups, W, scored):
    print(f"[reorder] {groups} {W} {scored}", flush=True)
    rng = np.random.default_rng(groups + W)
    n = groups * W
    lens = rng.integers(0, 200, n + 3).tolist()
    m = model(rng, lens, 16, 1, 64, spare=4)
    c = device_cache(m)
    score, want = scores_for(m, c, rng)
    for step in range(4):
        parent = rng.integers(0, W, (groups, W))
        slots = None if step == 0 else rng.permutation(n + 3)[:n].tolist()
        if step == 2:  # entries that do nothing
            parent[rng.random((groups, W)) < 0.2] = -1
            parent[rng.random((groups, W)) < 0.1] = W
            for i in range(n):
                if rng.random() < 0.2:
                    slots[i] = int(rng.integers(-2, n + 5))
        trevs.pages_reorder(c, dev(parent), None if slots is None else dev(slots), score=score if scored else None)
        do.reorder(m, parent.tolist(), slots, want if scored else None)
        check_table(c, m)
        assert np.array_equal(host(score), want)
    check_contents(c, m)


def test_reorder_then_reserve_gives_beams_their_own_last_page():
    rng = np.random.default_rng(2)
    m = model(rng, [37, 37, 37, 37], 16, 1, 64, spare=8, max_pages=4)
    c = device_cache(m)
    trevs.pages_reorder(c, dev([[2, 2, 0, 2]]))
    do.reorder(m, [[2, 2, 0, 2]])
    got = trevs.pages_reserve(c, dev([1] * 4))
    assert [t.tolist() for t in got] == [list(x) for x in m.reserve([1] * 4)]
    trevs.kv8_copy(c, got[1], got[2])
    m.copy(got[1].tolist(), got[2].tolist())
    check_table(c, m)
    check_contents(c, m)


# ------------------------------------------------------------------ together
class Decode:
    """Two prompts, each with three beams: head norms and rotation, rows written, attended to and
    scored in two layers, eviction down to a budget, the best continuations, sequences reordered."""

    def __init__(self, dtype, steps=7):
        rng = np.random.default_rng(21)
        self.B, self.W, self.P, self.V, self.steps = 2, 3, 75, 300, steps
        self.H_q, self.H_kv, self.d, self.page, self.budget = 8, 2, 64, 16, 60
        n = self.n = self.B * self.W
        t = lambda *s: storage(rng.normal(size=s), dtype)[0]  # noqa: E731
        self.cache = c = trevs.Kv8Cache(n_pages=120, page_tokens=self.page, n_slots=n, max_pages=8, H_kv=self.H_kv,
                                        d_head=self.d, n_layers=2)
        self.score = trevs.kv8_scores(c)
        w = [t(self.d), t(self.d)]
        kw = dict(freqs=trevs.rope_frequencies(self.d).cuda(), q_weight=w[0], k_weight=w[1], weight_offset=1.0)
        first = dev([0, self.W])
        pos = dev(np.broadcast_to(np.arange(self.P), (1, self.B, self.P)), torch.int64)
        self.norms, self.weighed, self.attended = [], [], []
        self.start = [trevs.PagesFree(c, dev(list(range(n)))), trevs.PagesReserve(c, dev([self.P] * 2), first)]
        for layer in range(2):
            norm = trevs.NormRope(t(self.B, self.P, self.H_q, self.d), t(self.B, self.P, self.H_kv, self.d), pos, **kw)
            attn = trevs.Kv8Attention(c, norm.q_out, slots=first, layer=layer, want_lse=True)
            self.start += [norm, trevs.Kv8Write(c, norm.k_out, t(self.B, self.P, self.H_kv, self.d), slots=first, layer=layer),
                           attn, trevs.Kv8Weights(c, norm.q_out, attn.lse, self.score, slots=first, layer=layer,
                                                  decay=float(layer))]
        # beams 1 and 2 take over from beam 0
        self.start.append(trevs.PagesReorder(c, dev([[0] * self.W] * 2), score=self.score))
        self.loop, self.selected, self.evicted = [], [], []
        beams, done = storage(np.array([[0.0, -math.inf, -math.inf]] * 2), torch.float32)[0], None
        ones = dev([1] * n)
        for i in range(steps):
            at = dev(np.full((1, n, 1), self.P + i), torch.int64)
            room = trevs.PagesReserve(c, ones)
            step = [room, trevs.Kv8Copy(c, room.copy_src, room.copy_dst)]
            for layer in range(2):
                norm = trevs.NormRope(t(n, 1, self.H_q, self.d), t(n, 1, self.H_kv, self.d), at, **kw)
                attn = trevs.Kv8Attention(c, norm.q_out, layer=layer, want_lse=True)
                step += [norm, trevs.Kv8Write(c, norm.k_out, t(n, 1, self.H_kv, self.d), layer=layer), attn,
                         trevs.Kv8Weights(c, norm.q_out, attn.lse, self.score, layer=layer, decay=1.0 - 0.25 * (layer == 0))]
                self.attended.append(attn)
            select = trevs.BeamSelect(t(self.B, self.W, self.V), beams, done, n_out=self.W, eos=1)
            evict = trevs.Kv8Evict(c, self.score, n_keep=self.budget, n_first=2, n_last=9)
            step += [select, trevs.PagesReorder(c, select.parent, score=self.score), evict]
            beams = select.score_out
            self.loop.append(step)
            self.selected.append(select)
            self.evicted.append(evict)

    def __call__(self):
        for call in self.start + [x for step in self.loop for x in step]:
            call()

    def outputs(self):
        c = self.cache
        return ([x for s in self.selected for x in (s.score_out, s.parent, s.token)]
                + [x for e in self.evicted for x in (e.n_evicted, e.kept_idx)]
                + [a.out for a in self.attended] + [self.score, c.len, c.ref, c.table])


@pytest.mark.parametrize("dtype", DTYPES)
def test_decode_run(dtype):
    """Every page call, selection and eviction of the run against the oracle's, which takes the device's
    own scores; attention over what is left against the oracle."""
    run = Decode(dtype)
    c = run.cache
    m = co.CacheModel(120, run.page, run.n, 8, run.H_kv, run.d, 2)
    run.score.fill_(math.nan)  # (decay 0 begins them anew; the other beams' come with the reordering)
    run.score[[1, 2, 4, 5]] = 0.0
    for call in run.start + [x for step in run.loop for x in step]:
        before = host(run.score).copy()
        call()
        if isinstance(call, trevs.PagesReserve):
            n_new, slots = call.inputs
            m.reserve(n_new.tolist(), None if slots is None else slots.tolist())
        elif isinstance(call, trevs.Kv8Copy):
            m.copy(call.inputs[0].tolist(), call.inputs[1].tolist())
        elif isinstance(call, trevs.Kv8Write):
            k, v, _, slots = call.inputs
            m.write(host(k), host(v), None, None if slots is None else slots.tolist(), call.args.layer)
        elif isinstance(call, trevs.Kv8Weights):
            q, lse, _, slots = call.inputs
            want = before.copy()
            slots = list(range(run.n)) if slots is None else slots.tolist()
            decay = float(call.args.decay)
            bound = do.weights(m, host(q), host(lse), want, None, slots, call.args.layer, decay=decay)
            check_weights(host(run.score)[slots], want[slots], *[x[slots] for x in bound], decay,
                          np.nan_to_num(before[slots]))
        elif isinstance(call, trevs.PagesReorder):
            want = before.copy()
            do.reorder(m, call.inputs[0].tolist(), None, want)
            assert np.array_equal(host(run.score), want)
        elif isinstance(call, trevs.Kv8Evict):
            want = before.copy()
            lists = do.evict(m, want, run.budget, 2, 9)
            assert [call.n_evicted.tolist(), call.kept_idx.tolist()] == [list(x) for x in lists]
            assert np.array_equal(host(run.score), want)
        elif isinstance(call, trevs.BeamSelect):
            x, s, _ = call.inputs
            check_beams((call.score_out, call.parent, call.token), host(x), host(s), None, run.W, 1)
        check_table(c, m)
    check_contents(c, m)
    assert max(m.len) == run.budget and m.ref.count(0) > 60


def test_decode_run_captured():
    """The run captured once and replayed: the same bits as the eager run, with eager work between."""
    run = Decode(torch.bfloat16, steps=4)
    run.score.zero_()
    run()
    torch.cuda.synchronize()
    want = [x.clone() for x in run.outputs()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(3):
        for x in run.outputs()[:-4]:
            x.fill_(3)
        run.score.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(run.outputs(), want):
            assert torch.equal(a, b), i
        if i == 1:  # eager calls between the replays
            run.score.zero_()
            run()
            torch.cuda.synchronize()
            for a, b in zip(run.outputs(), want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["norm", "weights", "evict", "beam", "reorder"])
def test_one_off_calls_on_another_stream(kind):
    """A one-off call on a given stream, its inputs dropped at once and memory taken by other work."""
    stream = torch.cuda.Stream()
    results = []
    for side in (None, stream):
        m = model(np.random.default_rng(30), [300, 200, 260, 90], 16, 2, 64, spare=60)
        c = device_cache(m)
        q, qs = storage(np.random.default_rng(1).normal(size=(4, 3, 4, 64)), torch.float32)
        score = scores_for(m, c, np.random.default_rng(2))[0]
        torch.cuda.synchronize()
        if kind == "norm":
            out = trevs.norm_rope(q, None, dev(np.zeros((1, 4, 3)), torch.int64), stream=side,
                                  freqs=dev(co.rope_frequencies(64), torch.float64))[0]
        elif kind == "weights":
            _, lse, _, _ = m.attention(qs)
            out = trevs.kv8_weights(c, q, storage(lse, torch.float32)[0], score, stream=side)
        elif kind == "evict":
            out = trevs.kv8_evict(c, score, stream=side, n_keep=80)
        elif kind == "beam":
            out = trevs.beam_select(storage(np.random.default_rng(3).normal(size=(4, 3, 9999)), torch.float32)[0],
                                    torch.zeros(4, 3, device="cuda"), stream=side, n_out=5)
        else:
            trevs.pages_reorder(c, dev([[1, 0], [1, 1]]), stream=side, score=score)
            out = score
        del q
        junk = [torch.full((1 << 18,), 7.0, device="cuda") for _ in range(8)]
        if side is not None:
            torch.cuda.current_stream().wait_stream(side)
        out = out if isinstance(out, tuple) else (out,)
        results.append([x.clone() for x in out] + [c.len.clone(), c.table.clone(), score.clone()])
        torch.cuda.synchronize()
        del junk
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_binding_refusals():
    q = torch.zeros(2, 3, 4, 64, device="cuda")
    pos, f = torch.zeros(1, 2, 3, dtype=torch.int64, device="cuda"), torch.zeros(32, dtype=torch.float64, device="cuda")
    w = torch.ones(64, device="cuda")
    for kw in (dict(q_weight=w[:32]), dict(q_weight=w.double()), dict(q_weight=torch.ones(3, 64, device="cuda")),
               dict(k_weight=w), dict(q_weight=w.cpu()), dict(q_weight=torch.ones(64, 2, device="cuda")[:, 0])):
        with pytest.raises((ValueError, TypeError)):
            trevs.NormRope(q, None, pos, freqs=f, **kw)
    with pytest.raises((ValueError, TypeError)):
        trevs.NormRope(q, q, pos, freqs=f, q_weight=w, k_weight=w.bfloat16())
    with pytest.raises(trevs.TrevsError):
        trevs.norm_rope(q, None, pos, freqs=f, eps=0.0)
    c = trevs.Kv8Cache(n_pages=4, page_tokens=16, n_slots=2, max_pages=2, H_kv=2, d_head=64)
    score = trevs.kv8_scores(c)
    lse = torch.zeros(2, 4, 3, device="cuda")
    for args in ((q, lse[:1], score), (q, lse, score[:1]), (q, lse, score.double()), (q.half(), lse, score),
                 (q[..., :32], lse, score), (q, lse.cpu(), score)):
        with pytest.raises((ValueError, TypeError)):
            trevs.Kv8Weights(c, *args)
    for kw in (dict(layer=1), dict(kv_max=33), dict(decay=-1.0), dict(scale=0.0)):
        with pytest.raises(trevs.TrevsError):
            trevs.Kv8Weights(c, q, lse, score, **kw)
    for kw in (dict(n_keep=0), dict(n_keep=5, n_first=3, n_last=3), dict(n_keep=5, n=3)):
        with pytest.raises(trevs.TrevsError):
            trevs.Kv8Evict(c, score, **kw)
    with pytest.raises(ValueError):
        trevs.Kv8Evict(c, score, dev([0, 1]), n_keep=5, keep=dev([1]))
    x, s = torch.zeros(2, 3, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    for args in ((x, s[:1]), (x, s.double()), (x.half(), s), (x.transpose(1, 2), s), (x, s, s)):
        with pytest.raises((ValueError, TypeError)):
            trevs.BeamSelect(*args, n_out=2)
    for kw in (dict(n_out=0), dict(n_out=65), dict(n_out=2, eos=50)):
        with pytest.raises(trevs.TrevsError):
            trevs.BeamSelect(x, s, **kw)
    with pytest.raises(trevs.TrevsError):
        trevs.pages_reorder(c, dev([[0, 1, 2]]))
    with pytest.raises((ValueError, TypeError)):
        trevs.PagesReorder(c, dev([[0, 1]]), dev([0]))
