"""Calls on a stream that is not torch's current one: what a call allocates must be safe to use there at once."""
import functools

import pytest

from test_gpu_block_select import ring

pytestmark = pytest.mark.gpu
BUSY = 60_000_000                                        # clocks that the current stream is kept busy: about 30 ms


def test_fresh_means_are_cleared_on_the_stream_that_fills_them():
    """The current stream still has work queued when the call comes: a clearing enqueued there would wipe the means."""
    import torch
    from paper_2603_17051_b200 import binding as A
    cache, _, _, _ = ring(A, 1, 2, 64, 50, 0, 5, 2, 4, 301)
    want = A.astro_block_pool(cache, 16)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    got = A.astro_block_pool(cache, 16, stream=side)
    torch.cuda.synchronize()
    assert want.any() and torch.equal(got, want)


@functools.lru_cache(maxsize=None)
def calls():
    """name -> (size in bytes of its first output, call on a stream)."""
    import torch
    from paper_2603_17051_b200 import binding as A
    B, n, H, D = 1, 4096, 16, 64
    g = torch.Generator(device="cuda").manual_seed(40)
    q, k, v, d_o = (torch.randn((B, m, H, D), generator=g, device="cuda").bfloat16() for m in (n, 512, 512, n))
    x = (q.flatten() * 8).view(1, -1)                     # 8 MB of velocities
    blocks = torch.arange(2, dtype=torch.int32, device="cuda").expand(B, H, n // 128, 2).contiguous()
    o, lse = A.astro_sparse_attn_fwd(None, q, k, v, blocks, 128, 0.125)
    delta = A.astro_chunk_attn_bwd_delta(o, d_o)
    rope = A.astro_rope_create(D, D, "halves", (32,))
    pos = torch.arange(n, dtype=torch.int32, device="cuda").view(1, n, 1)
    cache = A.astro_kvcache_create(B, H, D, n // 8, 0, 8)
    A.astro_kvcache_append(cache, q, d_o, 8)
    r = torch.full((1,), 0.5, device="cuda")
    size = q.numel() * 2
    return {
        "sparse forward": (size, lambda s: A.astro_sparse_attn_fwd(None, q, k, v, blocks, 128, 0.125, stream=s)),
        "sparse backward": (size, lambda s: A.astro_sparse_attn_bwd(None, q, k, v, blocks, 128, o, lse, d_o, 0.125, stream=s)),
        "rotary": (size, lambda s: A.astro_rope_apply(rope, q, None, pos, stream=s)[:1]),
        "dense forward": (size, lambda s: A.astro_chunk_attn_fwd(None, q, k, v, 0.125, stream=s)),
        "dense backward": (size, lambda s: A.astro_chunk_attn_bwd(None, q, k, v, o, lse, d_o, 0.125, stream=s)),
        "dense dq": (size, lambda s: (A.astro_chunk_attn_bwd_dq(None, q, k, v, lse, delta, d_o, 0.125, stream=s),)),
        "export": (size, lambda s: A.astro_kvcache_export(cache, stream=s)),
        "loss": (size, lambda s: A.astro_nft_loss(x, x, None, x, r, 0.5, stream=s)),
    }


@pytest.mark.parametrize("name", ["sparse forward", "sparse backward", "rotary", "dense forward", "dense backward", "dense dq",
                                  "export", "loss"])
def test_a_call_does_not_write_memory_that_queued_work_still_reads(name):
    """A tensor is dropped while the current stream still has a copy of it queued; a call on another stream must not be given
    its memory."""
    import torch
    size, call = calls()[name]
    want = [t for t in call(torch.cuda.current_stream()) if t is not None]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    victim = torch.ones(size, dtype=torch.uint8, device="cuda")
    copy = torch.zeros_like(victim)
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    copy.copy_(victim)
    del victim
    got = [t for t in call(side) if t is not None]
    torch.cuda.synchronize()
    assert (copy == 1).all()
    tight = 1e-5 if name == "loss" else 0.0               # its sums are atomic
    assert all(torch.allclose(a.float(), b.float(), rtol=tight, atol=0.0) for a, b in zip(want, got))


def test_what_a_call_returns_stays_whole_while_either_stream_uses_it():
    """A result made on another stream and read on the current one is dropped while the read is queued: the next calls on the other
    stream must not be given its memory."""
    import torch
    _, call = calls()["sparse forward"]
    side = torch.cuda.Stream()
    o, _ = call(side)
    torch.cuda.synchronize()
    want, copy = o.clone(), torch.zeros_like(o)
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    copy.copy_(o)
    del o
    for _ in range(3):
        with torch.cuda.stream(side):
            torch.empty_like(copy).zero_()
    torch.cuda.synchronize()
    assert torch.equal(copy, want)


def test_calls_on_a_stream_that_joined_a_capture():
    """Inside a captured graph, on a stream forked from the capturing one, with results dropped along the way."""
    import torch
    from paper_2603_17051_b200 import binding as A
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v, d_o = (torch.randn((1, n, 2, 64), generator=g, device="cuda").bfloat16() for n in (300, 256, 256, 300))
    blocks = torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda").expand(1, 2, 3, 3).contiguous()

    def whole(stream):
        o, lse = A.astro_sparse_attn_fwd(None, q, k, v, blocks, 64, 0.125, stream=stream)
        return (o, lse) + A.astro_sparse_attn_bwd(None, q, k, v, blocks, 64, o, lse, d_o, 0.125, stream=stream)

    want = [x.clone() for x in whole(None)]
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            out = whole(side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    A.astro_last_device_status()
    assert all(torch.equal(x, y) for x, y in zip(want, out))
