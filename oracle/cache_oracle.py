"""CPU oracle of the serving cache: rotary positions, the paged 8-bit K/V
cache, its page table and the attention over it, in float64 NumPy and plain
Python.  Test infrastructure only; shares no code with the HIP library.

A cache is a `CacheModel`: the e4m3 numbers of every block (as float64
values), the blocks' scales, and the page table.  Its methods serve requests
one after the other, which is what the library's page operations are defined
by.
"""

import math

import numpy as np


# ------------------------------------------------------------------ rotary
def rope_frequencies(rot_dim, base=10000.0, scaling="none", factor=1.0, original_len=0, beta_fast=32.0,
                     beta_slow=1.0):
    """Turns per position of each pair."""
    out = []
    for i in range(rot_dim // 2):
        f = base ** (-2.0 * i / rot_dim) / (2.0 * math.pi)
        if scaling == "linear":
            f = f / factor
        elif scaling == "parts":
            own = (original_len * f - beta_slow) / (beta_fast - beta_slow)
            own = min(max(own, 0.0), 1.0)
            f = own * f + (1.0 - own) * f / factor
        out.append(f)
    return np.array(out)


def rope(x, pos, freqs, sections, interleaved=False, inverse=False, attn_factor=1.0):
    """x [B,S,H,d] float64, pos [n_pos,B,S] int64, freqs [R/2] turns per position."""
    half = len(freqs)
    plane = np.repeat(np.arange(len(sections)), sections)
    assert len(plane) == half
    turns = np.stack([pos[plane[i]].astype(np.float64) * freqs[i] for i in range(half)], -1)
    w = 2.0 * math.pi * (turns - np.rint(turns)) * (-1.0 if inverse else 1.0)
    c, s = attn_factor * np.cos(w)[:, :, None], attn_factor * np.sin(w)[:, :, None]
    first = np.arange(half) * 2 if interleaved else np.arange(half)
    second = first + 1 if interleaved else first + half
    y = x.copy()
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    return y


# -------------------------------------------------------------- 8-bit blocks
def e4m3(x):
    """The e4m3 number nearest to x (ties to even), |x| <= 448."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(np.abs(x))  # |x| in [2^(e-1), 2^e)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)  # 3 fraction bits; subnormals share 2^-9
    return np.rint(x / step) * step


def block_scale(amax):
    """The smallest power of two s in 2^-126..2^120 with amax <= 448 s."""
    amax = np.asarray(amax, np.float64)
    out = np.full(amax.shape, 2.0 ** -126)
    for e in range(-126, 120):
        out = np.where(amax > 448.0 * 2.0 ** e, 2.0 ** (e + 1), out)
    return out


def e4m3_bytes():
    """The 256 numbers of the format by their byte (NaN for 0x7f and 0xff)."""
    out = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = math.nan if e == 15 and m == 7 else (m / 8.0 * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7))
        out[b] = -v if b & 128 else v
    return out


class CacheModel:
    def __init__(self, n_pages, page, n_slots, max_pages, H_kv, d, n_layers=1):
        self.page, self.max_pages, self.n_pages, self.n_slots = page, max_pages, n_pages, n_slots
        # numbers [L,n_pages,H,page,d] of keys and of values (token first here)
        self.k = np.zeros((n_layers, n_pages, H_kv, page, d))
        self.v = np.zeros((n_layers, n_pages, H_kv, page, d))
        self.k_scale = np.zeros((n_layers, n_pages, H_kv))
        self.v_scale = np.zeros((n_layers, n_pages, H_kv))
        self.table = [[-1] * max_pages for _ in range(n_slots)]
        self.len = [0] * n_slots
        self.ref = [0] * n_pages

    def _slot(self, s):
        return 0 <= s < self.n_slots

    def _pages(self, tokens):
        return -(-tokens // self.page)

    def _valid(self, p):
        return 0 <= p < self.n_pages

    # ---- page table
    def reserve(self, n_new, slots=None):
        slots = list(range(len(n_new))) if slots is None else list(slots)
        granted, src, dst = [], [], []
        for i, (s, n) in enumerate(zip(slots, n_new)):
            granted.append(0)
            src.append(-1)
            dst.append(-1)
            if not self._slot(s) or s in slots[:i] or n < 1 or self.len[s] + n > self.max_pages * self.page:
                continue
            have, want = self._pages(self.len[s]), self._pages(self.len[s] + n)
            last = self.table[s][have - 1] if self.len[s] % self.page else -1
            copy = self._valid(last) and self.ref[last] > 1
            free = [p for p in range(self.n_pages) if self.ref[p] == 0][:want - have + copy]
            if len(free) < want - have + copy:
                continue
            for p in free:
                self.ref[p] = 1
            if copy:
                self.ref[last] -= 1
                src[i], dst[i] = last, free[0]
            self.table[s][have - copy:want] = free
            self.len[s] += n
            granted[i] = n
        return granted, src, dst

    def fork(self, src, dst, n_tokens=None):
        done = []
        for i, (a, b) in enumerate(zip(src, dst)):
            ok = self._slot(a) and self._slot(b) and a not in dst and b not in dst[:i] and self.len[b] == 0
            done.append(int(ok))
            if not ok:
                continue
            n = self.len[a] if n_tokens is None else min(max(n_tokens[i], 0), self.len[a])
            for j in range(self._pages(n)):
                self.table[b][j] = p = self.table[a][j]
                if self._valid(p):
                    self.ref[p] += 1
            self.len[b] = n
        return done

    def free(self, slots, keep=None):
        slots = list(slots)
        for i, s in enumerate(slots):
            if not self._slot(s) or s in slots[:i]:
                continue
            n = 0 if keep is None else min(max(keep[i], 0), self.len[s])
            for j in range(self._pages(n), self._pages(self.len[s])):
                p = self.table[s][j]
                if self._valid(p):
                    self.ref[p] = max(self.ref[p] - 1, 0)
                self.table[s][j] = -1
            self.len[s] = n

    # ---- pages' contents
    def copy(self, src, dst):
        for a, b in zip(src, dst):
            if self._valid(a) and self._valid(b):
                for t in (self.k, self.v, self.k_scale, self.v_scale):
                    t[:, b] = t[:, a]

    def write(self, k, v, n_new=None, slots=None, layer=0):
        B, T = k.shape[:2]
        for b in range(B):
            s = b if slots is None else slots[b]
            if not self._slot(s):
                continue
            n = min(T if n_new is None else max(n_new[b], 0), T, self.len[s])
            start = self.len[s] - n
            for j in range(start // self.page, self._pages(self.len[s]) if n else 0):
                p = self.table[s][j]
                if not self._valid(p):
                    continue
                lo, hi = max(start - j * self.page, 0), min(self.len[s] - j * self.page, self.page)
                rows = slice(j * self.page + lo - start, j * self.page + hi - start)
                for x, data, scale in ((k, self.k, self.k_scale), (v, self.v, self.v_scale)):
                    new = x[b, rows].transpose(1, 0, 2)  # [H,n,d]
                    sc = block_scale(np.abs(new).max(axis=(1, 2)))
                    if lo:
                        old = scale[layer, p]
                        sc = np.maximum(sc, old)
                        data[layer, p, :, :lo] = e4m3(data[layer, p, :, :lo] * (old / sc)[:, None, None])
                    data[layer, p, :, lo:hi] = e4m3(new / sc[:, None, None])
                    scale[layer, p] = sc

    def compact(self, kept, src, dst, P, K_in):
        kept = np.asarray(kept)
        for b in range(len(src)):
            if not self._slot(src[b]) or not self._slot(dst[b]) or src[b] == dst[b]:
                continue
            L = self.len[src[b]]
            if L < P + K_in:
                continue
            rows = list(range(P)) + [P + min(max(int(i), 0), K_in - 1) for i in kept[b]] + list(range(P + K_in, L))
            rows = rows[:self.len[dst[b]]]
            for data, scale in ((self.k, self.k_scale), (self.v, self.v_scale)):
                vals = np.zeros((data.shape[0], data.shape[2], len(rows), data.shape[4]))
                for i, r in enumerate(rows):
                    p = self.table[src[b]][r // self.page]
                    if self._valid(p):
                        vals[:, :, i] = data[:, p, :, r % self.page] * scale[:, p][..., None]
                for j in range(self._pages(len(rows))):
                    p = self.table[dst[b]][j]
                    if not self._valid(p):
                        continue
                    part = vals[:, :, j * self.page:(j + 1) * self.page]
                    sc = block_scale(np.abs(part).max(axis=(2, 3)))
                    data[:, p, :, :part.shape[2]] = e4m3(part / sc[..., None, None])
                    scale[:, p] = sc

    def attention(self, q, q_len=None, slots=None, layer=0, causal=True, scale=None, kv_max=0):
        """Returns out [B,T,H_q,d] and lse [B,H_q,T] (NaN where no row is
        computed), and per row sum_j p_j |v_j| and the largest scale sum |q k_j|."""
        B, T, H_q, d = q.shape
        G = H_q // self.k.shape[2]
        scale = d ** -0.5 if scale is None else scale
        out = np.full(q.shape, math.nan)
        lse = np.full((B, H_q, T), math.nan)
        weight, size = np.zeros(q.shape), np.zeros((B, H_q, T))
        for b in range(B):
            s = b if slots is None else slots[b]
            m = min(T if q_len is None else max(q_len[b], 0), T)
            L = min(self.len[s], kv_max or self.max_pages * self.page) if self._slot(s) else 0
            there = np.array([self._valid(self.table[s][j // self.page]) for j in range(L)], bool)
            ids = [self.table[s][j // self.page] if there[j] else 0 for j in range(L)]
            at = np.arange(L) % self.page
            for h in range(H_q):
                g = h // G
                k = self.k[layer, ids, g, at] * self.k_scale[layer, ids, g][:, None] if L else np.zeros((0, d))
                v = self.v[layer, ids, g, at] * self.v_scale[layer, ids, g][:, None] if L else np.zeros((0, d))
                for t in range(m):
                    n = min(L - m + t + 1, L) if causal else L
                    use = np.nonzero(there[:max(n, 0)])[0]
                    out[b, t, h], lse[b, h, t] = 0.0, -math.inf
                    if len(use) == 0:
                        continue
                    x = scale * (k[use] @ q[b, t, h])
                    top = x.max()
                    p = np.exp(x - top)
                    lse[b, h, t] = top + math.log(p.sum())
                    p /= p.sum()
                    out[b, t, h] = p @ v[use]
                    weight[b, t, h] = p @ np.abs(v[use])
                    size[b, h, t] = scale * (np.abs(k[use]) @ np.abs(q[b, t, h])).max()
        return out, lse, weight, size
