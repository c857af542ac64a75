"""CPU oracle of the decode loop over the serving cache: head norms with the
rotation, attention weights summed for each cached token, eviction by them,
beam search's selection and the beams' sequences reordered; float64 NumPy and
plain Python over cache_oracle's CacheModel.  Test infrastructure only."""

import math

import numpy as np

from .cache_oracle import block_scale, e4m3, rope


def norm_rope(x, w, offset, eps, pos, freqs, sections, interleaved=False, attn_factor=1.0):
    """x [B,S,H,d]; w [d], [H,d] or None.  Returns the result and the normed values."""
    y = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    if w is not None:
        y = y * (w + offset)
    return rope(y, pos, freqs, sections, interleaved, False, attn_factor), y


def weights(m, q, lse, score, q_len=None, slots=None, layer=0, causal=True, scale=None, kv_max=0, decay=1.0):
    """score [n_slots, max_pages * page] updated in place.  Returns per token a
    bound's parts: the sum of its weights, of weight times the largest
    |scale q||k| + |logit| + |lse| that entered them, and their number."""
    B, T, H_q, d = q.shape
    G = H_q // m.k.shape[2]
    scale = d ** -0.5 if scale is None else scale
    total, spread, count = [np.zeros_like(score) for _ in range(3)]
    for b in range(B):
        s = b if slots is None else slots[b]
        if not 0 <= s < m.n_slots:
            continue
        rows = min(T if q_len is None else max(q_len[b], 0), T)
        L = min(max(m.len[s], 0), kv_max or m.max_pages * m.page, m.max_pages * m.page)
        if decay == 0.0:
            score[s] = 0.0
        score[s, :L] *= decay
        for j in range(L):
            p = m.table[s][j // m.page]
            if not 0 <= p < m.n_pages:
                continue
            # the first row that sees token j
            first = max(j - (L - rows), 0) if causal else 0
            if first >= rows:
                continue
            k = m.k[layer, p, :, j % m.page] * m.k_scale[layer, p][:, None]  # [H,d]
            k = np.repeat(k, G, 0)
            x = scale * np.einsum("thd,hd->ht", q[b, first:rows], k)
            z = lse[b, :, first:rows]
            with np.errstate(invalid="ignore"):
                e = np.where(np.isneginf(z) & ~np.isnan(x), 0.0, np.exp(x - z))
                size = scale * np.einsum("thd,hd->ht", np.abs(q[b, first:rows]), np.abs(k))
            total[s, j] = e.sum()
            spread[s, j] = (e * (size * (d + 8) + 4 * (np.abs(x) + np.abs(np.where(np.isinf(z), 0, z))))).sum()
            count[s, j] = e.size
            score[s, j] += total[s, j]
    return total, spread, count


def evict(m, score, n_keep, n_first=0, n_last=0, keep=None, slots=None, n=None):
    slots = list(range(n if n is not None else len(keep) if keep is not None else m.n_slots)) if slots is None \
        else list(slots)
    evicted, lists = [0] * len(slots), [[-1] * n_keep for _ in slots]
    free = [p for p in range(m.n_pages) if m.ref[p] <= 0]
    given_up = []
    for i, s in enumerate(slots):
        if not 0 <= s < m.n_slots or s in slots[:i]:
            continue
        L = min(max(m.len[s], 0), m.max_pages * m.page)
        n = n_keep if keep is None else min(max(keep[i], n_first + n_last, 1), n_keep)
        if L <= n:
            continue
        rank = [(math.inf if math.isnan(x) else -x, j) for j, x in enumerate(score[s][:L])]
        middle = sorted(rank[n_first:L - n_last])[:n - n_first - n_last]
        kept = list(range(n_first)) + sorted(j for _, j in middle) + list(range(L - n_last, L))
        assert len(kept) == n
        moved = next((a for a in range(n) if kept[a] != a), n)
        want = -(-n // m.page)
        start = moved // m.page if moved < n else want
        if want - start > len(free):
            continue
        old = list(m.table[s])
        for f in range(start, want):
            p = free.pop(0)
            m.ref[p], m.table[s][f] = 1, p
            part = kept[f * m.page:(f + 1) * m.page]
            for data, scale in ((m.k, m.k_scale), (m.v, m.v_scale)):
                x = np.zeros((data.shape[0], data.shape[2], len(part), data.shape[4]))
                for a, j in enumerate(part):
                    o = old[j // m.page]
                    if 0 <= o < m.n_pages:
                        x[:, :, a] = data[:, o, :, j % m.page] * scale[:, o][..., None]
                sc = block_scale(np.abs(x).max(axis=(2, 3)))
                data[:, p, :, :len(part)] = e4m3(x / sc[..., None, None])
                scale[:, p] = sc
        given_up += old[start:-(-L // m.page)]
        for f in range(want, -(-L // m.page)):
            m.table[s][f] = -1
        score[s][:n] = score[s][kept]
        score[s][n:L] = 0.0
        m.len[s] = n
        evicted[i], lists[i][:n] = L - n, kept
    for p in given_up:  # free for later calls only
        if 0 <= p < m.n_pages:
            m.ref[p] = max(m.ref[p] - 1, 0)
    return evicted, lists


def reorder(m, parent, slots=None, score=None):
    groups, W = len(parent), len(parent[0])
    slots = list(range(groups * W)) if slots is None else list(slots)
    ok = [0 <= s < m.n_slots and s not in slots[:i] for i, s in enumerate(slots)]
    table, length = [list(r) for r in m.table], list(m.len)
    was = None if score is None else score.copy()
    for i, s in enumerate(slots):
        p = parent[i // W][i % W]
        j = i // W * W + p
        if not ok[i] or not 0 <= p < W or not ok[j] or j == i:
            continue
        src = slots[j]
        n_old, n_new = [-(-min(max(length[x], 0), m.max_pages * m.page) // m.page) for x in (s, src)]
        for f in range(max(n_old, n_new)):
            now, old = table[src][f] if f < n_new else -1, table[s][f] if f < n_old else -1
            if 0 <= now < m.n_pages:
                m.ref[now] += 1
            if 0 <= old < m.n_pages:
                m.ref[old] -= 1
            m.table[s][f] = now
        m.len[s] = length[src]
        if score is not None:
            a, b = max(length[s], 0), max(length[src], 0)
            score[s, :b] = was[src, :b]
            score[s, b:a] = 0.0


def beam_select(logits, score, done, n_out, eos):
    """logits [B,W,V], score [B,W] (float64 values of what the call reads)."""
    B, W, V = logits.shape
    out = []
    for b in range(B):
        found = []
        for w in range(W):
            own = score[b, w] if score[b, w] < math.inf else -math.inf
            if done is not None and done[b, w]:
                found.append((-own, w, eos))
                continue
            x = logits[b, w]
            top = x.max() if not np.isnan(x).any() else math.nan
            if not np.isfinite(top) or not np.isfinite(own):
                found += [(math.inf, w, v) for v in range(min(n_out, V))]
                continue
            p = own + (x - top) - math.log(np.exp(x - top).sum())
            best = np.argsort(-p, kind="stable")[:n_out]
            found += [(-p[v], w, int(v)) for v in best]
        found.sort()
        out.append((found + [(math.inf, -1, -1)] * n_out)[:n_out])
    return (np.array([[-f[0] for f in r] for r in out]), np.array([[f[1] for f in r] for r in out]),
            np.array([[f[2] for f in r] for r in out]))
