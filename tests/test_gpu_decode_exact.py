"""The decode loop's results where they can be held to less than the general bounds allow: every rank of a
selection, logits of one product, a loop of beams that finish."""
import math

import numpy as np
import pytest
import torch

from oracle import decode_oracle as do
from paper_2609_37581_amd import trevs
from test_gpu_cache import dev, device_cache, host, model, storage
from test_gpu_decode import BEAMS, scores_for

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
TOL = 80 * 2.0 ** -24  # of a score before it is rounded, as in check_beams


def check_every_rank(got, x, s, done, n, eos):
    """Each returned score is that of the returned beam and token, nothing is returned twice, and what is not
    returned is no better than the last, by more than the bound."""
    score, parent, token = host(got[0]), got[1].cpu().numpy(), got[2].cpu().numpy()
    B, W, V = x.shape
    want, wp, wt = do.beam_select(x, s, done, n + 1, eos)
    for b in range(B):
        for r in range(n):
            w, v = int(parent[b, r]), int(token[b, r])
            if (w, v) == (-1, -1):
                assert (wp[b, r], wt[b, r]) == (-1, -1) and score[b, r] == -math.inf, (b, r)
                continue
            own = s[b, w] if s[b, w] < math.inf else -math.inf
            if done is not None and done[b, w]:
                assert v == eos
                exact = own
            else:
                top = x[b, w].max()
                exact = own + (x[b, w, v] - top) - math.log(np.exp(x[b, w] - top).sum()) if np.isfinite(top) else -math.inf
            assert score[b, r] == exact or abs(score[b, r] - exact) <= TOL + 2.0 ** -24 * abs(exact), (b, r, w, v)
            # as good as this rank's own, within what either is off by
            assert exact == want[b, r] or abs(exact - want[b, r]) <= 2 * TOL, (b, r, exact, want[b, r])
            near = [i for i in range(n + 1) if i != r and want[b, i] > -math.inf and abs(want[b, i] - want[b, r]) <= 2 * TOL
                    and wp[b, i] != wp[b, r]]
            if not near:
                assert (w, v) == (wp[b, r], wt[b, r]), (b, r)
        pairs = [p for p in zip(parent[b], token[b]) if p != (-1, -1)]
        assert len(set(pairs)) == len(pairs)
        assert all(a >= b for a, b in zip(score[b], score[b][1:]))


@pytest.mark.parametrize("shape", BEAMS + [(3, 1, 30000, 1, 1), (2, 8, 40001, 1, 0), (1, 64, 4099, 1, 3), (2, 3, 4096, 2, 0),
                                           (1, 2, 2049, 63, 1), (4, 16, 2048, 33, 0)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_beam_select_every_rank(shape, dtype):
    B, W, V, n, pad = shape
    print(f"[every rank] {shape} {dtype}", flush=True)
    rng = np.random.default_rng(2 * V + W)
    full, x = storage(rng.normal(size=(B, W, V + pad)) * 3, dtype)
    logits, x = full[:, :, :V], x[:, :, :V]
    score, s = storage(-3 * rng.random((B, W)), torch.float32)
    check_every_rank(trevs.beam_select(logits, score, n_out=n), x, s, None, n, 0)
    done = rng.random((B, W)) < 0.3
    eos = int(rng.integers(0, V))
    check_every_rank(trevs.beam_select(logits, score, dev(done), n_out=n, eos=eos), x, s, done, n, eos)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 3, 16, 64])
def test_beam_select_best_in_any_place(dtype, n):
    """The best lie next to each other, at a chunk's end, one to a chunk, or at the end of a row."""
    rng = np.random.default_rng(n)
    V = 20003
    x = rng.normal(size=(4, 2, V))
    for b, places in enumerate((range(4000, 4000 + n), range(4096 - n // 2, 4096 - n // 2 + n), range(5, V, V // n),
                                range(V - n, V))):
        for i, v in enumerate(list(places)[:n]):
            x[b, (i * 7) % 2, v] = 9.0 + 0.125 * ((i * 5) % 64)
    logits, x = storage(x, dtype)
    score, s = storage(np.array([[-0.25, -0.3125]] * 4), torch.float32)
    check_every_rank(trevs.beam_select(logits, score, n_out=n), x, s, None, n, 0)


@pytest.mark.parametrize("T,H_kv,d,max_pages", [(1, 1, 64, 0), (1, 2, 128, 512), (3, 1, 256, 0), (2, 10, 64, 512), (40, 2, 64, 0),
                                                (70, 1, 128, 0), (33, 1, 256, 0)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_weights_of_single_products(T, H_kv, d, max_pages, dtype):
    """Rows with one value each: a logit is one product, with all of the row's bits in it."""
    print(f"[single products] {T} {H_kv} {d} {max_pages} {dtype}", flush=True)
    rng = np.random.default_rng(T + d)
    B, G = 2, 2
    m = model(rng, [90, T + 3], 16, H_kv, d)
    if max_pages:
        m.table = [row + [-1] * (max_pages - len(row)) for row in m.table]
        m.max_pages = max_pages
    c = device_cache(m)
    scale = 0.125
    x = np.zeros((B, T, H_kv * G, d))
    at = rng.integers(0, d, x.shape[:3])
    for i in np.ndindex(*x.shape[:3]):
        b, _, h = i
        pages = m.table[b][:-(-m.len[b] // 16)]
        k = m.k[0, pages, h // G, :, at[i]] * m.k_scale[0, pages, h // G][:, None]
        x[i][at[i]] = (20 + 10 * rng.random()) * rng.choice([-1, 1]) / (scale * np.abs(k).max())
    q, qs = storage(x, dtype)
    _, lse, _, _ = m.attention(qs, scale=scale)
    ld, ls = storage(lse, torch.float32)
    score, want = scores_for(m, c, rng)
    old = want.copy()
    total, short, bound = [np.zeros_like(want) for _ in range(3)]
    two = q.bfloat16().float() + (q.float() - q.bfloat16().float()).bfloat16().float()
    two = host(two)  # the rows in two parts
    for i in np.ndindex(*x.shape[:3]):
        b, t, h = i
        n = m.len[b] - T + t + 1
        j = np.arange(n)
        page = np.array(m.table[b])[j // 16]
        z = scale * qs[i][at[i]] * m.k[0, page, h // G, j % 16, at[i]] * m.k_scale[0, page, h // G]
        e = np.exp(z - ls[b, h, t])
        total[b, :n] += e
        short[b, :n] += np.exp(z * (two[i][at[i]] / qs[i][at[i]]) - ls[b, h, t])
        # the sum of a logit's parts twice, the scale, its product with log2 e and a block's scale, and the difference's
        # rounding, 2^-24 each (log2 e's own cancels where the two are equal: once more for each); the exponential 2^-22
        bound[b, :n] += e * ((8 * np.abs(z) + 3 * abs(ls[b, h, t])) * 2.0 ** -24 + 2.0 ** -22)
    want += total
    bound += (T * H_kv * G + 4) * 2.0 ** -24 * (total + bound) + 2.0 ** -23 * (np.abs(old) + np.abs(want))
    assert dtype == torch.bfloat16 or (np.abs(short - total) > 2 * bound).any()  # a lost third part shows
    trevs.kv8_weights(c, q, ld, score, scale=scale)
    err = np.abs(host(score) - want)
    assert np.all(err <= bound), (err / np.maximum(bound, 1e-300)).max()


def test_beams_that_finish():
    """A loop that goes on until its beams have ended, `done` following the beams: against a search that keeps
    whole sequences."""
    rng = np.random.default_rng(17)
    B, W, V, eos, steps = 3, 4, 11, 2, 9
    table, x = storage(rng.normal(size=(V, V)) * 2 + 1.5 * (np.arange(V) == eos), torch.float32)  # logits after a token
    table_lp = x - np.log(np.exp(x).sum(-1, keepdims=True))
    beam = torch.full((B, W), -math.inf, device="cuda")
    beam[:, 0] = 0.0
    token = dev(rng.integers(3, V, (B, 1))).expand(B, W).contiguous()
    start = token[:, 0].tolist()
    done = torch.zeros(B, W, dtype=torch.int32, device="cuda")
    seqs = [[[] for _ in range(W)] for _ in range(B)]
    plain = [[(0.0, [], False)] for _ in range(B)]
    for _ in range(steps):
        logits = table[token.clamp(min=0).long()]
        beam, parent, token = trevs.beam_select(logits, beam, done, n_out=W, eos=eos)
        done = done.gather(1, parent.clamp(min=0).long()) | (token == eos).int()
        seqs = [[seqs[b][p] + [t] for p, t in zip(parent[b].tolist(), token[b].tolist())] for b in range(B)]
        for b in range(B):
            more = []
            for s, seq, over in plain[b]:
                last = seq[-1] if seq else start[b]
                more += [(s, seq + [eos], True)] if over else [(s + table_lp[last, v], seq + [v], v == eos) for v in range(V)]
            plain[b] = sorted(more, key=lambda c: -c[0])[:W]
            gaps = [p[0] - q[0] for p, q in zip(plain[b], plain[b][1:])]
            assert min(gaps) > 1e-4  # (no rank is in doubt)
    for b in range(B):
        assert seqs[b] == [seq for _, seq, _ in plain[b]]
        assert done[b].tolist() == [int(over) for _, _, over in plain[b]]
        assert np.abs(host(beam[b]) - [s for s, _, _ in plain[b]]).max() <= steps * (TOL + 2.0 ** -24 * 40)
    assert done.all()
