"""Timed cases of the decode loop over the serving cache: head norms with the
rotation, attention weights summed up for each cached token and the eviction
by them, and beam search with its sequences reordered.

`run` computes a pass either in plain torch operations (own = False) or
through the entry points of paper_2609_37581_amd.trevs (own = True), on the
same inputs.  A case is a dict of plain values; `kind` names the operator:

  norm     RMS norms of the heads of queries and keys, then their rotary
           positions (trevs.NormRope)
  weights  the attention weights that query rows give to each cached token,
           added to the tokens' scores (trevs.Kv8Weights)
  evict    cached sequences cut down to the tokens of the highest scores
           (trevs.Kv8Evict)
  beam     the best continuations over beams and vocabulary (trevs.BeamSelect)
  reorder  the beams' sequences taken over from their parents
           (trevs.PagesReorder)

The cache holds e4m3 values and one power-of-two scale for each page of
tokens and KV head: k [pages, H_kv, page, d], v [pages, H_kv, d, page],
scales [pages, H_kv]; scores are float32 [slots, tokens of the table].  Sizes
are those of the workloads in synthetic/workloads.py (LLaVA-1.5-7B,
LLaVA-NeXT-7B and Qwen2.5-VL-7B shapes) and generic odd ones.
"""

import math

import torch

own = False

F8 = torch.float8_e4m3fn

# ----------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------


def listed():
    return [
        # q and k of a batch of pruned long images, three position planes
        dict(name="norm-prompt-qwen", kind="norm", dtype="bf16", B=4, S=4259, H_q=28, H_kv=4, d=128, rot=128, n_pos=3,
             inter=False, per_head=False, offset=0.0, far=16384),
        # one decode step of a served batch far into a long context: latency, part of the head, a weight a head
        dict(name="norm-token-f32", kind="norm", dtype="f32", B=64, S=1, H_q=32, H_kv=32, d=128, rot=64, n_pos=1,
             inter=True, per_head=True, offset=1.0, far=1000000),
        # one decode step of an interactive chat in fp32: launches and latency
        dict(name="weights-token-b1-f32", kind="weights", dtype="f32", B=1, T=1, ragged=False, lo=259, hi=259, H_q=32,
             H_kv=32, d=128, page=16, causal=True, decay=1.0),
        # one decode step of a served batch over long visual contexts
        dict(name="weights-token-b64", kind="weights", dtype="bf16", B=64, T=1, ragged=False, lo=1187, hi=16547,
             H_q=28, H_kv=4, d=128, page=64, causal=True, decay=0.98),
        # what questions of 32 to 128 rows look at in their long images
        dict(name="weights-question-b8", kind="weights", dtype="bf16", B=8, T=128, ragged=True, lo=16451, hi=16547,
             H_q=28, H_kv=4, d=128, page=32, causal=True, decay=0.0),
        # what the pruned prompts of a batch of long images look at
        dict(name="weights-prompt-qwen", kind="weights", dtype="bf16", B=4, T=4259, ragged=False, lo=4259, hi=4259,
             H_q=28, H_kv=4, d=128, page=64, causal=True, decay=0.0),
        # long contexts of a served batch cut to a budget
        dict(name="evict-qwen", kind="evict", B=4, lo=4259, hi=16547, keep=2048, ragged=False, first=4, last=256,
             H_kv=4, d=128, page=64, layers=4),
        # many short contexts, some within their budget already
        dict(name="evict-llava15-b64", kind="evict", B=64, lo=131, hi=700, keep=256, ragged=True, first=4, last=32,
             H_kv=32, d=128, page=16, layers=1),
        # a step of one chat with four beams in fp32: latency
        dict(name="beam-b1-f32", kind="beam", dtype="f32", B=1, W=4, V=32000, n_out=8, finished=False, banned=False,
             pad=0),
        # a step of a served batch with a large vocabulary, finished beams and banned tokens among them
        dict(name="beam-b64", kind="beam", dtype="bf16", B=64, W=8, V=152064, n_out=16, finished=True, banned=True,
             pad=0),
        # the beams of one chat
        dict(name="reorder-chat", kind="reorder", B=1, W=4, lo=259, hi=259, T=20, page=16, scored=False),
        # the beams of a served batch of long images, with the scores of their tokens
        dict(name="reorder-serve", kind="reorder", B=16, W=8, lo=1187, hi=16547, T=100, page=64, scored=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "weights", "weights", "weights", "evict", "evict", "beam", "beam", "reorder"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    H_q, H_kv, d = rng.choice(((32, 32, 128), (28, 4, 128), (32, 8, 128), (16, 16, 64), (8, 1, 256)))
    page = rng.choice((16, 32, 64))
    if kind == "norm":
        S = rng.choice((1, _log_int(rng, 2, 4259)))
        B = _log_int(rng, 1, max(1, min(64, 16384 // S)))
        return dict(kind="norm", dtype=dtype, B=B, S=S, H_q=H_q, H_kv=H_kv, d=d, rot=rng.choice((d, d, d // 2, 48)),
                    n_pos=rng.choice((1, 3)), inter=rng.random() < 0.5, per_head=rng.random() < 0.5,
                    offset=rng.choice((0.0, 1.0)), far=_log_int(rng, 4096, 1000000))
    if kind == "weights":
        form = rng.choice(("token", "chunk", "prompt"))
        if form == "prompt":
            T = lo = hi = _log_int(rng, 32, 4259 if dtype == "bf16" else 2048)
            B = _log_int(rng, 1, max(1, min(16, 16384 // T)))
        else:
            T = 1 if form == "token" else rng.randint(2, 128)
            lo = T + _log_int(rng, 16, 8192)
            hi = lo + rng.randint(0, 8192)
            B = _log_int(rng, 1, 64 if form == "token" else 8)
        return dict(kind="weights", dtype=dtype, B=B, T=T, ragged=form == "chunk", lo=lo, hi=hi, H_q=H_q, H_kv=H_kv,
                    d=d, page=page, causal=rng.random() < 0.75, decay=rng.choice((0.0, 0.95, 1.0)))
    if kind == "evict":
        keep = _log_int(rng, 24, 2048)
        lo = _log_int(rng, max(1, keep // 2), 4 * keep)
        first = rng.randint(0, min(8, keep // 8))
        return dict(kind="evict", B=_log_int(rng, 1, max(1, min(64, 8192 // keep))), lo=lo,
                    hi=lo + _log_int(rng, 1, 4 * keep), keep=keep, ragged=rng.random() < 0.5, first=first,
                    last=rng.randint(0, keep // 2 - first), H_kv=H_kv, d=d, page=page,
                    layers=rng.randint(1, 4 if H_kv <= 8 else 1))
    if kind == "beam":
        V = _log_int(rng, 500, 152064)
        W = rng.randint(1, 8)
        return dict(kind="beam", dtype=dtype, B=_log_int(rng, 1, 64 if dtype == "bf16" else 32), W=W, V=V,
                    n_out=W * rng.randint(1, 2), finished=rng.random() < 0.5, banned=rng.random() < 0.5,
                    pad=rng.choice((0, 0, 1, 64)))
    lo = _log_int(rng, 40, 4096)
    return dict(kind="reorder", B=_log_int(rng, 1, 16), W=rng.randint(2, 8), lo=lo, hi=lo + rng.randint(0, 8192),
                T=rng.randint(1, 200), page=page, scored=rng.random() < 0.5)


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------


def _spread(n, lo, hi):
    """n lengths spread evenly over lo..hi."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]


def _ceil(a, b):
    return -(-a // b)


class _Draws:
    def __init__(self, case, seed):
        self.dev = torch.device("cuda")
        self.gen = torch.Generator(self.dev).manual_seed(seed & 0x7fffffff)
        self.host = torch.Generator().manual_seed(seed & 0x7fffffff)
        self.dt = torch.bfloat16 if case.get("dtype") == "bf16" else torch.float32

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device=self.dev, dtype=torch.float32)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.gen, device=self.dev, dtype=torch.float32)

    def perm(self, n):
        return torch.randperm(n, generator=self.host).tolist()

    def ints(self, values):
        return torch.tensor(values, dtype=torch.int32, device=self.dev)

    def keys(self, *shape):
        """Key or value rows [..., d]: N(0,1) with a few strong channels, as projections have them."""
        x = self.normal(*shape)
        gain = torch.ones(shape[-1], device=self.dev)
        gain[self.perm(shape[-1])[:max(1, shape[-1] // 32)]] = 4.0
        return x * gain


def _lengths(c):
    return _spread(c["B"], c["lo"], c["hi"])


def _query_lengths(c):
    return _spread(c["B"], max(1, c["T"] // 4), c["T"]) if c.get("ragged") else [c["T"]] * c["B"]


def _filled(r, layers, n_pages, H, page, d):
    """A cache whose every page holds quantised rows."""
    k = torch.empty((layers, n_pages, H, page, d), device=r.dev, dtype=F8)
    v = torch.empty((layers, n_pages, H, d, page), device=r.dev, dtype=F8)
    ks = torch.empty((layers, n_pages, H), device=r.dev)
    vs = torch.empty((layers, n_pages, H), device=r.dev)
    for layer in range(layers):
        x, y = r.keys(n_pages, H, page, d), r.keys(n_pages, H, page, d)
        # levels differ from page to page, so the scales do too
        x *= torch.exp2(r.normal(n_pages, 1, 1, 1).clamp(-2, 2) * 0.5)
        y *= torch.exp2(r.normal(n_pages, 1, 1, 1))
        ks[layer], vs[layer] = _pow2_scale(x.abs().amax((2, 3))), _pow2_scale(y.abs().amax((2, 3)))
        k[layer] = (x / ks[layer][:, :, None, None]).to(F8)
        v[layer] = (y / vs[layer][:, :, None, None]).to(F8).transpose(2, 3)
    return k, v, ks, vs


def _tables(r, slots_pages, max_pages, spare):
    """Page lists of the sequences, drawn without order from all pages."""
    n = sum(slots_pages) + spare
    order = r.perm(n)
    rows, at = [], 0
    for m in slots_pages:
        rows.append(order[at:at + m] + [-1] * (max_pages - m))
        at += m
    return rows, n


def _counts(rows, n_pages):
    ref = [0] * n_pages
    for row in rows:
        for p in row:
            if p >= 0:
                ref[p] += 1
    return ref


def _scores(r, lens, width):
    """Summed weights: a heavy tail, the first tokens of a sequence far above the others, zeros past its end."""
    s = torch.exp(2.0 * r.normal(len(lens), width)) * 1e-2
    s[:, :4] *= 50.0
    return s * (torch.arange(width, device=r.dev) < r.ints(lens)[:, None])


def _norm_inputs(c, seed):
    r = _Draws(c, seed)
    B, S, d = c["B"], c["S"], c["d"]
    # heads of different levels, a few strong channels
    level = torch.exp2(torch.linspace(-2, 3, c["H_q"] + c["H_kv"], device=r.dev))[:, None]
    q = (r.keys(B, S, c["H_q"], d) * level[:c["H_q"]]).to(r.dt)
    k = (r.keys(B, S, c["H_kv"], d) * level[c["H_q"]:]).to(r.dt)
    start = torch.randint(0, max(1, c["far"] - S), (c["n_pos"], B, 1), generator=r.host)
    pos = (start + torch.arange(S)).to(r.dev)
    w = [(1.0 - c["offset"] + 0.3 * r.normal(*((H, d) if c["per_head"] else (d,)))).to(r.dt)
         for H in (c["H_q"], c["H_kv"])]
    return r, q, k, pos, w[0], w[1]


EPS = 1e-6
BASE = 500000.0


def _sections(c):
    half = c["rot"] // 2
    a = half // 4
    b = (half - a) // 2
    return [half] if c["n_pos"] == 1 else [a, b, half - a - b]


def _weights_inputs(c, seed):
    r = _Draws(c, seed)
    page = c["page"]
    lens = [_lengths(c)[i] for i in r.perm(c["B"])]
    pages = [_ceil(n, page) for n in lens]
    rows, n_pages = _tables(r, pages, max(pages), max(2, sum(pages) // 16))
    k, v, ks, vs = _filled(r, 1, n_pages, c["H_kv"], page, c["d"])
    beta = torch.linspace(0.5, 2.0, c["H_q"], device=r.dev)[:, None]
    q = (r.normal(c["B"], c["T"], c["H_q"], c["d"]) * beta).to(r.dt)
    score = _scores(r, lens, max(pages) * page)
    s = dict(k=k, v=v, ks=ks, vs=vs, table=r.ints(rows), len=r.ints(lens), ref=r.ints(_counts(rows, n_pages)),
             n_pages=n_pages, max_pages=max(pages), lens=lens, q=q, q_len=r.ints(_query_lengths(c)), first=score,
             score=score.clone())
    # the log-sum-exp that the layer's attention over the cache left
    lse = torch.zeros((c["B"], c["H_q"], c["T"]), device=r.dev)
    for b, x in _logits(c, s):
        lse[b:b + x.shape[0]] = torch.logsumexp(x, -1).reshape(x.shape[0], c["H_q"], c["T"])
    s["lse"] = lse
    return r, s


def _evict_inputs(c, seed):
    r = _Draws(c, seed)
    page = c["page"]
    lens = [_lengths(c)[i] for i in r.perm(c["B"])]
    pages = [_ceil(n, page) for n in lens]
    rows, n_pages = _tables(r, pages, max(pages), c["B"] * _ceil(c["keep"], page))
    k, v, ks, vs = _filled(r, c["layers"], n_pages, c["H_kv"], page, c["d"])
    least = max(c["first"] + c["last"], 1)
    keep = _spread(c["B"], max(least, c["keep"] // 2), c["keep"]) if c["ragged"] else [c["keep"]] * c["B"]
    return r, dict(k=k, v=v, ks=ks, vs=vs, table=r.ints(rows), len=r.ints(lens), ref=r.ints(_counts(rows, n_pages)),
                   n_pages=n_pages, max_pages=max(pages), score=_scores(r, lens, max(pages) * page), keep=r.ints(keep))


def _beam_inputs(c, seed):
    r = _Draws(c, seed)
    B, W, V = c["B"], c["W"], c["V"]
    # a few likely tokens above the noise of the others
    x = 2.0 * r.normal(B, W, V + c["pad"])
    x += 8.0 * (r.uniform(B, W, V + c["pad"]) < 20.0 / V)
    if c["banned"]:
        x[:, :, r.perm(V)[:max(1, V // 100)]] = -math.inf
    logits = x.to(r.dt)
    if c["pad"]:
        logits = logits[:, :, :V]
    score = -20.0 * r.uniform(B, W)
    done = (r.uniform(B, W) < 0.2).to(torch.int32) if c["finished"] else None
    return r, dict(logits=logits, score=score, done=done)


def _reorder_inputs(c, seed):
    """The W beams of each sequence share the pages of its image and hold those of their own answers."""
    r = _Draws(c, seed)
    B, W, page = c["B"], c["W"], c["page"]
    lens = [_lengths(c)[i] for i in r.perm(B)]
    shared = [n // page for n in lens]
    total = [_ceil(n + c["T"], page) for n in lens]
    max_pages = max(total)
    own_pages = [t - s for t, s in zip(total, shared) for _ in range(W)]
    rows, n_pages = _tables(r, shared + own_pages, max_pages, 8)
    table = []
    for b in range(B):
        for w in range(W):
            mine = rows[B + b * W + w][:total[b] - shared[b]]
            table.append((rows[b][:shared[b]] + mine + [-1] * max_pages)[:max_pages])
    length = [n + c["T"] for n in lens for _ in range(W)]
    parent = torch.randint(0, W, (B, W), generator=r.host).tolist()
    s = dict(table=r.ints(table), len=r.ints(length), ref=r.ints(_counts(table, n_pages)), n_pages=n_pages,
             max_pages=max_pages, parent=r.ints(parent))
    if c["scored"]:
        s["score"] = _scores(r, length, max_pages * page)
    return r, s


def _cache_of(c, s, names):
    """The framework's cache with the state's contents, whose tensors take the place of the state's."""
    from paper_2609_37581_amd import trevs
    layers = s["k"].shape[0] if "k" in s else 1
    cache = trevs.Kv8Cache(n_pages=s["n_pages"], page_tokens=c["page"], n_slots=s["table"].shape[0],
                           max_pages=s["max_pages"], H_kv=c.get("H_kv", 1), d_head=c.get("d", 64), n_layers=layers)
    if "k" in s:
        for name, to in (("k", cache.k), ("v", cache.v)):
            to.copy_(s[name].view(torch.uint8))
            s[name] = to.view(F8)
    for name in names:
        to = dict(ks=cache.k_scale, vs=cache.v_scale, table=cache.table, len=cache.len, ref=cache.ref)[name]
        to.copy_(s[name])
        s[name] = to
    return cache


def prepare(case, seed):
    c = case
    if c["kind"] == "norm":
        r, q, k, pos, wq, wk = _norm_inputs(c, seed)
        s = dict(case=c, q=q, k=k, pos=pos, wq=wq, wk=wk)
        if own:
            from paper_2609_37581_amd import trevs
            freqs = trevs.rope_frequencies(c["rot"], base=BASE).to(r.dev)
            s["call"] = trevs.NormRope(q, k, pos, freqs=freqs, q_weight=wq, k_weight=wk, eps=EPS,
                                       weight_offset=c["offset"], sections=_sections(c), interleaved=c["inter"])
        return s
    if c["kind"] == "beam":
        _, s = _beam_inputs(c, seed)
        s["case"] = c
        if own:
            from paper_2609_37581_amd import trevs
            s["call"] = trevs.BeamSelect(s["logits"], s["score"], s["done"], n_out=c["n_out"], eos=2)
        return s
    if c["kind"] == "weights":
        _, s = _weights_inputs(c, seed)
        s["case"] = c
        if own:
            from paper_2609_37581_amd import trevs
            cache = _cache_of(c, s, ("ks", "vs", "table", "len", "ref"))
            s["call"] = trevs.Kv8Weights(cache, s["q"], s["lse"], s["score"], s["q_len"], causal=c["causal"],
                                         kv_max=max(s["lens"]), decay=c["decay"])
        return s
    _, s = (_evict_inputs if c["kind"] == "evict" else _reorder_inputs)(c, seed)
    s["case"] = c
    s["first"] = {n: s[n].clone() for n in ("table", "len", "ref", "score") if n in s}
    if own:
        from paper_2609_37581_amd import trevs
        if c["kind"] == "evict":
            cache = _cache_of(c, s, ("ks", "vs", "table", "len", "ref"))
            s["call"] = trevs.Kv8Evict(cache, s["score"], n_keep=c["keep"], n_first=c["first"], n_last=c["last"],
                                       keep=s["keep"] if c["ragged"] else None)
        else:
            cache = _cache_of(c, s, ("table", "len", "ref"))
            s["call"] = trevs.PagesReorder(cache, s["parent"], score=s.get("score"))
    return s


# ----------------------------------------------------------------------------
# plain forms
# ----------------------------------------------------------------------------


def _pow2_scale(amax):
    """The smallest power of two s with amax <= 448 s, at least 2^-126."""
    m, e = torch.frexp(amax)  # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(-126, 120)
    return torch.ldexp(torch.ones_like(amax), e)


def _plain_norm(s):
    c = s["case"]
    half, dev = c["rot"] // 2, s["q"].device
    f = BASE ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
    plane = torch.repeat_interleave(torch.arange(c["n_pos"], device=dev), torch.tensor(_sections(c), device=dev),
                                    output_size=half)
    angle = s["pos"][plane].permute(1, 2, 0).double() * f  # [B,S,half]
    cos, sin = [t.float()[:, :, None] for t in (angle.cos(), angle.sin())]

    def turn(x, w):
        y = x.float()
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * (w.float() + c["offset"])
        rot, rest = y[..., :c["rot"]], y[..., c["rot"]:]
        if c["inter"]:
            a, b = rot[..., 0::2], rot[..., 1::2]
            z = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = rot[..., :half], rot[..., half:]
            z = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return torch.cat((z, rest), -1).to(x.dtype)

    return dict(q=turn(s["q"], s["wq"]), k=turn(s["k"], s["wk"]))


def _logits(c, s):
    """The masked logits of a few sequences at a time: their first index, [m,H_kv,G*T,n] in 32 bits."""
    B, T, H_q, H_kv, d, page = c["B"], c["T"], c["H_q"], c["H_kv"], c["d"], c["page"]
    G, dev = H_q // H_kv, s["q"].device
    n = s["max_pages"] * page
    j, t = torch.arange(n, device=dev), torch.arange(T, device=dev)
    step = max(1, min(B, (1 << 29) // (H_q * T * n + H_kv * n * d)))
    for b in range(0, B, step):
        ids = s["table"][b:b + step].long().clamp(min=0)
        k = s["k"][0].view(torch.uint8)[ids].view(F8).float() * s["ks"][0][ids][..., None, None]
        m = ids.shape[0]
        kt = k.permute(0, 2, 4, 1, 3).reshape(m, H_kv, d, n)
        q = s["q"][b:b + step].float().reshape(m, T, H_kv, G, d).permute(0, 2, 3, 1, 4).reshape(m, H_kv, G * T, d)
        x = torch.matmul(q, kt).reshape(m, H_kv, G, T, n) * d ** -0.5
        kv, ql = s["len"][b:b + step, None, None], s["q_len"][b:b + step, None, None]
        seen = j < kv
        if c["causal"]:
            seen = seen & (j <= kv - ql + t[:, None])
        yield b, x.masked_fill_(~seen.expand(m, T, n)[:, None, None], -math.inf)


def _plain_weights(s):
    c = s["case"]
    B, T, H_q, H_kv = c["B"], c["T"], c["H_q"], c["H_kv"]
    n = s["score"].shape[1]
    j, t = torch.arange(n, device=s["q"].device), torch.arange(T, device=s["q"].device)
    for b, x in _logits(c, s):
        m = x.shape[0]
        live = t < s["q_len"][b:b + m, None]
        lse = s["lse"][b:b + m].reshape(m, H_kv, H_q // H_kv, T)
        w = (x - lse[..., None]).exp_() * live[:, None, None, :, None]
        w = w.sum(3).sum((1, 2))
        inside = j < s["len"][b:b + m, None]
        was = s["score"][b:b + m]
        now = (torch.zeros_like(w) if c["decay"] == 0.0 else c["decay"] * was) + w
        past = torch.zeros_like(was) if c["decay"] == 0.0 else was
        s["score"][b:b + m] = torch.where(inside, now, past)
    return dict(score=s["score"])


def _plain_evict(s):
    c = s["case"]
    B, page, n_keep, dev = c["B"], c["page"], c["keep"], s["k"].device
    table, length, ref, score = s["table"], s["len"], s["ref"], s["score"]
    n = score.shape[1]
    j = torch.arange(n, device=dev)
    L = length[:, None].long()
    budget = s["keep"].long()[:, None] if c["ragged"] else torch.full_like(L, n_keep)
    cut = (L > budget)[:, 0]
    held = (j < c["first"]) | (j >= L - c["last"])
    rank = torch.where(held, math.inf, score)
    rank = torch.where(j < L, rank, -math.inf)
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :n_keep]
    if order.shape[1] < n_keep:  # more than the table holds
        order = torch.nn.functional.pad(order, (0, n_keep - order.shape[1]), value=n)
    col = torch.arange(n_keep, device=dev)
    kept = torch.sort(torch.where(col < budget, order, n), dim=1).values  # ascending, n past the budget
    same = (kept == col).long().cumprod(1).sum(1)  # leading tokens that stay where they are
    live = budget[:, 0]
    first = torch.where(same == live, (live + page - 1) // page, same // page)
    have, want = (L[:, 0] + page - 1) // page, (live + page - 1) // page
    need = torch.where(cut, want - first, 0)
    free = torch.sort((ref > 0).to(torch.int32), stable=True).indices
    off = torch.cumsum(need, 0) - need
    pc = torch.arange(s["max_pages"], device=dev)
    old = table.long()
    take = cut[:, None] & (pc >= first[:, None]) & (pc < want[:, None])
    got = free[(off[:, None] + pc - first[:, None]).clamp(0, s["n_pages"] - 1)]
    gone = cut[:, None] & (pc >= first[:, None]) & (pc < have[:, None])
    # rows into the new pages, each block with a scale of its own
    width = _ceil(n_keep, page)
    seq, at = torch.nonzero(take[:, :width], as_tuple=True)
    rows = kept.gather(1, (torch.arange(width * page, device=dev) % (width * page)).clamp(max=n_keep - 1).expand(B, -1))
    rows = rows.reshape(B, width, page)[seq, at]  # [m,page]
    tok = at[:, None] * page + torch.arange(page, device=dev)
    real = tok < live[seq][:, None]
    rows = torch.where(real, rows, 0)
    src = old[seq].gather(1, rows // page).clamp(min=0)
    dst = got[seq, at]
    for pages, scales, flip in ((s["k"], s["ks"], False), (s["v"], s["vs"], True)):
        raw = pages.view(torch.uint8)
        for layer in range(c["layers"]):
            x = raw[layer].transpose(2, 3) if flip else raw[layer]
            x = x[src, :, rows % page].view(F8).float() * scales[layer][src][..., None]  # [m,page,H,d]
            x = x.transpose(1, 2) * real[:, None, :, None]
            s_new = _pow2_scale(x.abs().amax((2, 3)))
            y = (x / s_new[..., None, None]).to(F8).view(torch.uint8)
            y = y.transpose(2, 3) if flip else y
            mask = real[:, None, None, :] if flip else real[:, None, :, None]
            raw[layer][dst] = torch.where(mask, y, raw[layer][dst])
            scales[layer][dst] = s_new
    # the table, the counts, the lengths and the scores
    tally = torch.zeros(s["n_pages"] + 1, dtype=torch.int32, device=dev)
    tally.index_add_(0, torch.where(gone, old, s["n_pages"]).flatten(), torch.full_like(old.flatten(), -1, dtype=torch.int32))
    tally.index_add_(0, torch.where(take, got, s["n_pages"]).flatten(), torch.ones_like(old.flatten(), dtype=torch.int32))
    ref.add_(tally[:s["n_pages"]])
    table.copy_(torch.where(take, got, torch.where(gone, -1, old)))
    moved = torch.zeros_like(score)
    moved[:, :n_keep] = torch.where(col < budget, score.gather(1, kept.clamp(max=n - 1)), 0.0)[:, :n]
    score.copy_(torch.where(cut[:, None], moved, score))
    evicted = torch.where(cut, L[:, 0] - live, 0).to(torch.int32)
    length.copy_(torch.where(cut, live, L[:, 0]))
    kept = torch.where(cut[:, None] & (col < budget), kept, -1).to(torch.int32)
    return dict(n_evicted=evicted, kept_idx=kept)


def _plain_beam(s):
    c = s["case"]
    B, W, V, n_out = c["B"], c["W"], c["V"], c["n_out"]
    x = s["logits"].double()  # (in 64 bits: candidates of different beams may lie close together)
    top = x.amax(-1, keepdim=True)
    x = x - top
    x = x - x.exp().sum(-1, keepdim=True).log() + s["score"].double()[..., None]
    if s["done"] is not None:  # a finished beam goes on as it is
        fin = (s["done"] != 0)[..., None]
        only = torch.where(torch.arange(V, device=x.device) == 2, s["score"].double()[..., None], math.nan)
        x = torch.where(fin, only, x)
    x = x.reshape(B, W * V)
    there = ~x.isnan()
    best, at = torch.sort(torch.where(there, x, -math.inf), dim=1, descending=True, stable=True)
    best, at = best[:, :n_out], at[:, :n_out]
    short = ~there.gather(1, at)
    return dict(score=torch.where(short, -math.inf, best).float(),
                parent=torch.where(short, -1, at // V).to(torch.int32),
                token=torch.where(short, -1, at % V).to(torch.int32))


def _plain_reorder(s):
    c = s["case"]
    B, W = c["B"], c["W"]
    dev = s["table"].device
    src = (torch.arange(B, device=dev)[:, None] * W + s["parent"].long()).flatten()
    old, new = s["table"].clone(), s["table"][src]
    tally = torch.zeros(s["n_pages"] + 1, dtype=torch.int32, device=dev)
    for rows, sign in ((old, -1), (new, 1)):
        flat = torch.where(rows < 0, s["n_pages"], rows).long().flatten()
        tally.index_add_(0, flat, torch.full_like(flat, sign, dtype=torch.int32))
    s["ref"].add_(tally[:s["n_pages"]])
    s["table"].copy_(new)
    s["len"].copy_(s["len"][src])
    if c["scored"]:
        s["score"].copy_(s["score"][src])
    return {}


_PLAIN = dict(norm=_plain_norm, weights=_plain_weights, evict=_plain_evict, beam=_plain_beam, reorder=_plain_reorder)


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------


def run(state):
    s = state
    kind = s["case"]["kind"]
    if kind == "weights":
        s["score"].copy_(s["first"])  # the scores as they were before the pass
    elif kind in ("evict", "reorder"):  # and the page lists
        for name, was in s["first"].items():
            s[name].copy_(was)
    if not own:
        out = _PLAIN[kind](s)
    elif kind == "norm":
        q, k = s["call"]()
        out = dict(q=q, k=k)
    elif kind == "weights":
        s["call"]()
        out = dict(score=s["score"])
    elif kind == "evict":
        n_evicted, kept_idx = s["call"]()
        out = dict(n_evicted=n_evicted, kept_idx=kept_idx)
    elif kind == "beam":
        score, parent, token = s["call"]()
        out = dict(score=score, parent=parent, token=token)
    else:
        s["call"]()
        out = {}
    if kind == "evict":
        out.update(k=s["k"], v=s["v"], k_scale=s["ks"], v_scale=s["vs"])
    if kind in ("evict", "reorder"):
        out.update({name: s[name] for name in s["first"]})
    return out


def work(case):
    """Every input read once, every output written once, and the products of the visible pairs."""
    c = case
    e = 2 if c.get("dtype") == "bf16" else 4
    if c["kind"] == "norm":
        heads = c["H_q"] + c["H_kv"]
        values = c["B"] * c["S"] * heads * c["d"]
        return dict(bytes=2 * values * e + 8 * c["n_pos"] * c["B"] * c["S"]
                    + (heads if c["per_head"] else 2) * c["d"] * e,
                    flops=4 * values + 3 * values * c["rot"] // c["d"])
    if c["kind"] == "weights":
        lens, ql = _lengths(c), _query_lengths(c)
        rows = sum(ql) * c["H_q"]
        pairs = c["H_q"] * sum(q * (n - (q - 1) / 2 if c["causal"] else n) for n, q in zip(lens, ql))
        return dict(bytes=rows * (c["d"] * e + 4) + sum(lens) * (c["H_kv"] * (c["d"] + 4 / c["page"])
                                                                 + (8 if c["decay"] else 4)),
                    flops=2 * c["d"] * pairs)
    if c["kind"] == "evict":
        least = max(c["first"] + c["last"], 1)
        keep = _spread(c["B"], max(least, c["keep"] // 2), c["keep"]) if c["ragged"] else [c["keep"]] * c["B"]
        lens = _lengths(c)
        rows = sum(m for n, m in zip(lens, keep) if n > m)
        return dict(bytes=4 * sum(lens) + 12 * rows + rows * c["layers"] * c["H_kv"] * 4 * (c["d"] + 4 / c["page"]),
                    flops=2 * rows * c["layers"] * c["H_kv"] * c["d"])
    if c["kind"] == "beam":
        values = c["B"] * c["W"] * c["V"] * (0.8 if c["finished"] else 1.0)
        return dict(bytes=values * e + 8 * c["B"] * c["W"] + 12 * c["B"] * c["n_out"], flops=4 * values)
    tokens = c["W"] * (sum(_lengths(c)) + c["B"] * c["T"])
    return dict(bytes=8 * tokens // c["page"] + (8 * tokens if c["scored"] else 0) + 12 * c["B"] * c["W"], flops=0)


# ----------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------


def _e4m3(x):
    """Nearest e4m3 value (ties to even) of float64 values within +-448."""
    _, e = torch.frexp(x.abs())
    step = torch.exp2((e - 4).clamp(min=-9).double())  # 3 fraction bits, subnormals below 2^-6
    return torch.round(x / step) * step


def _block_scale(amax):
    e = torch.ceil(torch.log2(torch.where(amax > 0, amax, 1e-300) / 448.0))
    e = e - (torch.exp2(e - 1) * 448.0 >= amax).double() + (torch.exp2(e) * 448.0 < amax).double()
    return torch.exp2(e.clamp(-126, 120))


def _exact_norm(c, seed):
    _, q, k, pos, wq, wk = _norm_inputs(c, seed)
    half = c["rot"] // 2
    plane = [p for p, n in enumerate(_sections(c)) for _ in range(n)]
    angle = torch.stack([pos[plane[i]].double() * BASE ** (-2.0 * i / c["rot"]) for i in range(half)], -1)[:, :, None]
    out = {}
    for name, x, w in (("q", q, wq), ("k", k, wk)):
        y = x.double()
        rms = torch.sqrt(torch.sum(y ** 2, -1, keepdim=True) / c["d"] + EPS)
        y = y / rms * (w.double() + c["offset"])
        i = torch.arange(half, device=y.device)
        at_a, at_b = (2 * i, 2 * i + 1) if c["inter"] else (i, i + half)
        a, b = y[..., at_a], y[..., at_b]
        y[..., at_a] = a * angle.cos() - b * angle.sin()
        y[..., at_b] = a * angle.sin() + b * angle.cos()
        out[name] = y
    return out


def _exact_weights(c, seed):
    _, s = _weights_inputs(c, seed)
    page, G, d = c["page"], c["H_q"] // c["H_kv"], c["d"]
    q_len, table = s["q_len"].tolist(), s["table"].tolist()
    out = s["first"].double() * c["decay"]
    for b, n in enumerate(s["lens"]):
        m = q_len[b]
        if c["decay"]:
            out[b, n:] = s["first"][b, n:].double()
        ids = table[b][:_ceil(n, page)]
        for h in range(c["H_kv"]):
            k = s["k"][0, :, h].view(torch.uint8)[ids].view(F8).double() * s["ks"][0, ids, h, None, None].double()
            k = k.reshape(-1, d)[:n]
            for g in range(G):
                x = s["q"][b, :m, h * G + g].double() @ k.T / math.sqrt(d)
                if c["causal"]:
                    x += torch.full((m, n), -math.inf, dtype=torch.float64, device=x.device).triu(n - m + 1)
                out[b, :n] += torch.exp(x - s["lse"][b, h * G + g, :m, None].double()).sum(0)
    return dict(score=out)


def _exact_evict(c, seed):
    _, s = _evict_inputs(c, seed)
    page, B, n_keep = c["page"], c["B"], c["keep"]
    lens, table, ref = s["len"].tolist(), s["table"].tolist(), s["ref"].tolist()
    keep = s["keep"].tolist() if c["ragged"] else [n_keep] * B
    out = dict(k=s["k"].double(), v=s["v"].double(), k_scale=s["ks"].double(), v_scale=s["vs"].double())
    before = {name: t.clone() for name, t in out.items()}
    score = s["score"].cpu()
    evicted, kept_idx = [0] * B, [[-1] * n_keep for _ in range(B)]
    free = [p for p, n in enumerate(ref) if n == 0]
    for b in range(B):
        L, n = lens[b], keep[b]
        if L <= n:
            continue
        value = score[b].tolist()
        middle = sorted(range(c["first"], L - c["last"]), key=lambda i: (-value[i], i))
        kept = (list(range(c["first"])) + sorted(middle[:n - c["first"] - c["last"]]) + list(range(L - c["last"], L)))
        moved = next((i for i in range(n) if kept[i] != i), n)
        start = moved // page if moved < n else _ceil(n, page)
        row = list(table[b])
        for f in range(start, _ceil(n, page)):
            p = free.pop(0)
            ref[p], table[b][f] = 1, p
            part = kept[f * page:(f + 1) * page]
            src, at = [row[i // page] for i in part], [i % page for i in part]
            for name in ("k", "v"):
                data = before[name] if name == "k" else before[name].transpose(3, 4)
                x = data[:, src, :, at]  # [n,layers,H,d]
                x = x * before[name + "_scale"][:, src].transpose(0, 1)[..., None]
                x = x.permute(1, 2, 0, 3)  # [layers,H,n,d]
                scale = _block_scale(x.abs().amax((2, 3)))
                to = out[name] if name == "k" else out[name].transpose(3, 4)
                to[:, p, :, :len(part)] = _e4m3(x / scale[..., None, None])
                out[name + "_scale"][:, p] = scale
        for f in range(start, _ceil(L, page)):
            ref[row[f]] -= 1
            if f >= _ceil(n, page):
                table[b][f] = -1
        kept_idx[b][:n] = kept
        score[b] = torch.tensor([value[i] for i in kept] + [0.0] * (score.shape[1] - n))
        evicted[b], lens[b] = L - n, n
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(n_evicted=ints(evicted), kept_idx=ints(kept_idx), **out, table=ints(table), len=ints(lens),
                ref=ints(ref), score=score.double().cuda())


def _exact_beam(c, seed):
    _, s = _beam_inputs(c, seed)
    B, W, V, n_out = c["B"], c["W"], c["V"], c["n_out"]
    scores, parents, tokens = [], [], []
    for b in range(B):
        found = []
        for w in range(W):
            own_score = float(s["score"][b, w])
            if s["done"] is not None and int(s["done"][b, w]):
                found.append((-own_score, w, 2))
                continue
            p = torch.log_softmax(s["logits"][b, w].double(), 0) + own_score
            n = min(n_out, V)
            least = torch.topk(p, n).values[-1]
            at = torch.nonzero(p >= least)[:, 0] if torch.isfinite(least) else torch.arange(V, device=p.device)
            found += [(-x, w, t) for x, t in zip(p[at].tolist(), at.tolist())]
        found = (sorted(found) + [(math.inf, -1, -1)] * n_out)[:n_out]
        scores.append([-f[0] for f in found])
        parents.append([f[1] for f in found])
        tokens.append([f[2] for f in found])
    return dict(score=torch.tensor(scores, dtype=torch.float64, device="cuda"),
                parent=torch.tensor(parents, dtype=torch.int32, device="cuda"),
                token=torch.tensor(tokens, dtype=torch.int32, device="cuda"))


def _exact_reorder(c, seed):
    _, s = _reorder_inputs(c, seed)
    W = c["W"]
    table, length, parent = s["table"].tolist(), s["len"].tolist(), s["parent"].tolist()
    src = [b * W + parent[b][w] for b in range(c["B"]) for w in range(W)]
    rows = [table[i] for i in src]
    out = dict(table=rows, len=[length[i] for i in src], ref=_counts(rows, s["n_pages"]))
    out = {n: torch.tensor(x, dtype=torch.int32, device="cuda") for n, x in out.items()}
    if c["scored"]:
        out["score"] = torch.stack([s["score"][i] for i in src]).double()
    return out


def exact(case, seed):
    return dict(norm=_exact_norm, weights=_exact_weights, evict=_exact_evict, beam=_exact_beam,
                reorder=_exact_reorder)[case["kind"]](case, seed)
