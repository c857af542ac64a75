"""Attention over the cache planned for more keys than its sequences hold: the
workspace's contents never count, whatever calls came before, and one handle
serves sequences that grow, eager and replayed."""
import numpy as np
import pytest
import torch

from paper_2609_37581_amd import trevs
from test_gpu_cache import check_attention, check_table, dev, device_cache, model, storage

pytestmark = pytest.mark.gpu


def lengthened(m, max_pages):
    """The model with a longer table: its calls are planned for what that could hold."""
    m.table = [row + [-1] * (max_pages - len(row)) for row in m.table]
    m.max_pages = max_pages
    return m


def fill(call, value):
    call.workspace.view(torch.float32).fill_(value)
    call.out.fill_(7.0)
    call.lse.fill_(7.0)


LOOSE = [  # page, max_pages, H_q, H_kv, d, T, lens, q_len, causal, kv_max
    (64, 300, 28, 4, 128, 1, [1187], None, True, 0),               # a decode step over a long table
    (64, 300, 28, 4, 128, 1, [1187, 1216, 3, 64], None, True, 0),
    (16, 256, 32, 32, 128, 1, [259], None, True, 4096),
    (64, 512, 8, 8, 64, 1, [1000], None, True, 0),
    (32, 512, 16, 2, 256, 1, [500, 0, 129], None, True, 0),
    (32, 42, 8, 1, 256, 69, [1168, 1291], [69, 50], True, 1291),   # bounded exactly, but ragged and causal
    (64, 300, 28, 4, 128, 40, [500, 77], [40, 3], True, 0),
    (16, 2048, 6, 2, 64, 3, [90, 33, 1], None, False, 0),
    (16, 4096, 8, 4, 64, 64, [70], None, True, 0),
]


@pytest.mark.parametrize("shape", LOOSE)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_workspace_contents_do_not_count(shape, dtype):
    page, max_pages, H_q, H_kv, d, T, lens, q_len, causal, kv_max = shape
    print(f"[attn loose] {shape} {dtype}", flush=True)
    rng = np.random.default_rng(sum(lens))
    m = lengthened(model(rng, lens, page, H_kv, d), max_pages)
    c = device_cache(m)
    q, qs = storage(rng.normal(size=(len(lens), T, H_q, d)), dtype)
    call = trevs.Kv8Attention(c, q, None if q_len is None else dev(q_len), causal=causal, kv_max=kv_max, want_lse=True)
    first = None
    for value in (float("nan"), 3e4, -1.0, 0.0):
        fill(call, value)
        call()
        torch.cuda.synchronize()
        if first is None:
            check_attention(m, c, qs, call.out, call.lse, dtype, q_len=q_len, causal=causal, kv_max=kv_max)
            first = call.out.clone(), call.lse.clone()
        assert torch.equal(call.out, first[0]) and torch.equal(call.lse, first[1]), value
    # another call's sums, of logits far larger
    q.mul_(64.0)
    call()
    q.mul_(1 / 64.0)
    call.out.fill_(7.0)
    call.lse.fill_(7.0)
    call()
    torch.cuda.synchronize()
    assert torch.equal(call.out, first[0]) and torch.equal(call.lse, first[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("captured", [False, True])
def test_one_handle_while_sequences_grow(dtype, captured):
    """Decode steps through one set of handles, no bound given; captured, each
    replay against the eager definition."""
    print(f"[attn grow] {dtype} {captured}", flush=True)
    rng = np.random.default_rng(31)
    B, H_q, H_kv, d, page = 4, 14, 2, 128, 64
    m = lengthened(model(rng, [1214, 63, 640, 1], page, H_kv, d, spare=8), 300)
    c = device_cache(m)
    rows = [storage(rng.normal(size=(B, 1, H, d)), dtype) for H in (H_q, H_kv, H_kv)]
    (q, _), (k, _), (v, _) = rows
    room = trevs.PagesReserve(c, dev([1] * B))
    write = trevs.Kv8Write(c, k, v, room.granted)
    attn = trevs.Kv8Attention(c, q, want_lse=True)
    fill(attn, float("nan"))

    def step():
        room()
        write()
        attn()

    graph = None
    if captured:
        step()  # (loaded before it is captured)
        torch.cuda.synchronize()
        m = lengthened(model(np.random.default_rng(31), [1214, 63, 640, 1], page, H_kv, d, spare=8), 300)
        put(room.cache, m)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    for i in range(5):
        xs = [storage(rng.normal(size=t.shape), dtype) for t, _ in rows]
        for (t, _), (x, _) in zip(rows, xs):
            t.copy_(x)
        attn.out.fill_(7.0)
        attn.lse.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        assert m.reserve([1] * B)[0] == [1] * B
        m.write(xs[1][1], xs[2][1])
        check_table(room.cache, m)
        check_attention(m, room.cache, xs[0][1], attn.out, attn.lse, dtype)


def put(c, m):
    """A model's contents into a cache that handles refer to."""
    fresh = device_cache(m)
    for name in ("k", "v", "k_scale", "v_scale", "table", "len", "ref"):
        getattr(c, name).copy_(getattr(fresh, name))
