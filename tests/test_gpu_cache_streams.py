"""The one-off functions on a stream that is not the current one: what they
drop on return, and what the caller drops, is not reused while the stream still
works with it."""
import numpy as np
import pytest
import torch

from paper_2609_37581_amd import trevs
from test_gpu_cache import dev, device_cache, model, storage

pytestmark = pytest.mark.gpu


def behind(stream):
    """The stream waits for what is enqueued, then holds its work back for some 20 ms."""
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        torch.cuda._sleep(50_000_000)


def overwrite(like):
    """Memory of these sizes, freed on the current stream, is taken and overwritten."""
    for _ in range(4):
        held = [torch.full((t,), 0xFF, dtype=torch.uint8, device="cuda") for t in like]
        del held


@pytest.fixture
def sizes():
    """Bytes of everything that the binding allocates (without guard bands: blocks go back when dropped)."""
    seen = []

    def alloc(shape, dtype, device):
        t = torch.empty(shape, dtype=dtype, device=device)
        seen.append(t.numel() * t.element_size())
        return t

    before = trevs.set_allocator(alloc)
    yield seen
    trevs.set_allocator(before)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_on_another_stream(dtype, sizes):
    rng = np.random.default_rng(1)
    m = model(rng, [3000, 500], 64, 2, 128)
    c = device_cache(m)
    q, _ = storage(rng.normal(size=(2, 1, 8, 128)), dtype)
    q_len, slots = dev([1, 1]), dev([0, 1])
    want, want_lse = trevs.kv8_attention(c, q, q_len, slots, want_lse=True)
    torch.cuda.synchronize()
    for _ in range(2):
        side = torch.cuda.Stream()
        args = q.clone(), q_len.clone(), slots.clone()
        del sizes[:]
        behind(side)
        out, lse = trevs.kv8_attention(c, *args, stream=side, want_lse=True)
        taken = sizes + [t.numel() * t.element_size() for t in args]
        del args
        overwrite(taken)
        torch.cuda.current_stream().wait_stream(side)
        a, b = out.clone(), lse.clone()
        del out, lse
        with torch.cuda.stream(side):
            overwrite(taken)
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, want_lse)


def test_rotation_write_and_pages_on_another_stream(sizes):
    rng = np.random.default_rng(2)
    B, T, H, d, page = 3, 40, 2, 64, 16
    q, _ = storage(rng.normal(size=(B, T, H, d)), torch.bfloat16)
    pos, freqs = dev(rng.integers(0, 999, (1, B, T)), torch.int64), trevs.rope_frequencies(d).cuda()
    lists = [dev(x) for x in ([T, T - 3, 5], [0, 1, 2], [3, 4, 5])]
    kept = dev([[0, 3], [1, 2]])

    def run(stream, clone):
        c = trevs.Kv8Cache(n_pages=40, page_tokens=page, n_slots=6, max_pages=6, H_kv=H, d_head=d)
        out = []
        if stream is not None:
            behind(stream)
        for f in (lambda g: trevs.pages_reserve(c, g(lists[0]), g(lists[1]), stream=stream),
                  lambda g: trevs.rope(g(q), g(q), g(pos), freqs=g(freqs), stream=stream),
                  lambda g: trevs.kv8_write(c, g(q), g(q), g(lists[0]), g(lists[1]), stream=stream),
                  lambda g: trevs.pages_fork(c, g(lists[1]), g(lists[2]), stream=stream),
                  lambda g: trevs.pages_free(c, g(lists[2]), g(lists[1]), stream=stream),
                  lambda g: trevs.kv8_compact(c, g(kept), g(lists[1][:2].clone()), g(dev([4, 5])), P=0, K_in=4,
                                              stream=stream),
                  lambda g: trevs.kv8_copy(c, g(lists[1]), g(dev([30, 31, 32])), stream=stream)):
            del sizes[:]
            args = []

            def given(t):
                args.append(t.numel() * t.element_size())
                return t.clone() if clone else t

            r = f(given)
            if clone:
                overwrite(sizes + args)
            out += list(r) if isinstance(r, tuple) else [] if r is None else [r]
        torch.cuda.synchronize()
        return out + [c.k, c.v, c.k_scale, c.v_scale, c.len, c.ref]

    want = run(None, False)
    got = run(torch.cuda.Stream(), True)
    assert len(want) == len(got) and all(torch.equal(a, b) for a, b in zip(want, got))


def test_a_cache_that_is_dropped(sizes):
    rng = np.random.default_rng(3)
    m = model(rng, [2000], 32, 2, 128)
    c = device_cache(m)
    q, _ = storage(rng.normal(size=(1, 1, 4, 128)), torch.bfloat16)
    want = trevs.kv8_attention(c, q)
    torch.cuda.synchronize()
    del sizes[:]
    c = device_cache(m)
    taken = list(sizes)
    side = torch.cuda.Stream()
    behind(side)
    out = trevs.kv8_attention(c, q, stream=side)
    del c
    overwrite(taken)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_a_stream_of_another_device_is_refused():
    class Other:
        device = torch.device("cuda", 99)
        cuda_stream = 0

    c = trevs.Kv8Cache(n_pages=4, page_tokens=16, n_slots=2, max_pages=2, H_kv=1, d_head=64)
    with pytest.raises(ValueError):
        trevs.pages_reserve(c, dev([1, 1]), stream=Other())
