"""Refusals that need no device: handles that are gone, whole numbers beyond the C types, strides beyond any memory, frequencies
that are no numbers."""
import ctypes as C

import pytest

from paper_2603_17051_b200 import binding as A
from test_ops_abi_cpu import SHAPE, desc


def host_cache(**kw):
    """A cache over host memory: enough for everything that launches nothing."""
    import torch
    size = dict(cache_batch=1, heads=2, head_dim=64, tokens_per_frame=16, sink_frames=1, window_frames=4)
    size.update(kw)
    n = A.astro_kvcache_storage_bytes(*size.values())
    room = lambda: torch.empty(n, dtype=torch.uint8)  # noqa: E731
    return A.astro_kvcache_create(*size.values(), k_storage=room(), v_storage=room())


def test_a_destroyed_cache_is_not_an_empty_context():
    cache = host_cache()
    assert A.astro_block_count(cache, 100, 64) == (0, 2) and A.astro_kvcache_key_segments(cache, 5) == [(0, 5, 1)]
    A.astro_kvcache_destroy(cache)
    for call in (lambda: A.astro_block_count(cache, 100, 64), lambda: A.astro_kvcache_key_segments(cache, 5), lambda: A._handle(cache, -1),
                 lambda: A._cache(cache)):
        with pytest.raises(ValueError):
            call()
    A.astro_kvcache_destroy(cache)                         # again: nothing left to do
