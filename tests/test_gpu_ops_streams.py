"""Calls on a stream that is not torch's current one: what a call allocates must be safe to use there at once."""
import pytest

from helpers import dev_bf16
from paper_2603_17051_b200 import synth
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
