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


def test_whole_numbers_beyond_the_c_types_are_refused_not_cut():
    far = 2 ** 32
    for n_kc, block in ((100, far + 64), (far + 100, 64), (100, -far + 64)):
        with pytest.raises(A.AstroError) as e:
            A.astro_block_count(None, n_kc, block)
        assert e.value.status == SHAPE
    for f in ([0, far], [far + 1], [-far]):
        assert min(A._frame_list(f)[0]) < 0                # no frame, which the call refuses
    arr, n = A._frame_list([3, 0, 2 ** 31 - 1])
    assert n == 3 and list(arr)[:3] == [3, 0, 2 ** 31 - 1]
    assert A._frame_list(None) == (None, -1) and A._frame_list([])[1] == 0
    for size in (A.astro_block_select_workspace_bytes(1, 2, 64, 300, 40, far + 16), A.astro_sparse_attn_fwd_workspace_bytes(1, 2, 64, 5, far + 64, 128),
                 A.astro_sparse_attn_bwd_workspace_bytes(1, 2, 64, 300, 40, 4, far + 16)):
        assert size == 0                                   # as for every size that the calls refuse


def test_rotary_descriptions_beyond_the_c_types():
    for bad in (dict(head_dim=2 ** 32 + 64), dict(rot_dim=2 ** 32 + 64), dict(axis_pairs=(2 ** 32 + 32,))):
        with pytest.raises(A.AstroError) as e:
            A.astro_rope_create(**{**dict(head_dim=64, rot_dim=64, layout="halves", axis_pairs=(32,), scaling="linear", factor=2.0), **bad})
        assert e.value.status == SHAPE


@pytest.mark.parametrize("axes", [(1,), (0, 40), (-1,), [2 ** 32]])
def test_scaled_axes_that_are_not_there(axes):
    with pytest.raises(A.AstroError) as e:
        A.astro_rope_create(64, 64, "halves", (32,), scaling="linear", factor=2.0, scaled_axes=axes)
    assert e.value.status == SHAPE


def test_scaled_axes_may_come_from_an_iterator_and_name_any_axis():
    rope = A.astro_rope_create(64, 64, "halves", (16, 16), scaling="linear", factor=2.0, scaled_axes=iter((1,)))
    f = A.astro_rope_frequencies(rope)[0]
    assert f[0] == 1.0 and f[16] == 0.5


@pytest.mark.parametrize("bad", [dict(base=5e-324), dict(base=1e-300, scaling=2, factor=1e300), dict(magnitude=1e39), dict(magnitude=1e-46),
                                 dict(scaling=2, base=1e200, factor=1e200)])
def test_tables_that_are_no_numbers_are_refused(bad):
    """Frequencies or a magnitude that overflow would turn every position, 0 included, into NaN."""
    import math
    out = C.c_void_p()
    status = A.lib().astro_rope_create(C.byref(desc(**{**dict(scaled_axes=1), **bad})), C.byref(out))
    if status == 0:                                        # what is accepted is a table of numbers
        f, m = (C.c_double * 32)(), C.c_double()
        assert A.lib().astro_rope_frequencies(out, f, C.byref(m)) == 0
        assert all(0.0 < x < math.inf for x in f) and 0 < C.c_float(m.value).value < math.inf
        A.lib().astro_rope_destroy(out)
    else:
        assert status == SHAPE and not out.value


def test_strides_whose_products_pass_64_bits():
    """Output rows 2^40 elements apart, 2^29 of them: the second sample starts inside the first whatever 64-bit products say."""
    keep = A.astro_rope_create(64, 64, "halves", (32,))
    p = C.c_void_p
    strides = lambda *x: C.byref(A.Strides(*x))  # noqa: E731
    run = lambda si, so: A.lib().astro_rope_apply(keep.handle, 0, p(0x10000), None, p(0x30000), 1, 2, 1 << 29, 4, 0, 0, strides(*si),  # noqa: E731
                                                  p(0x40000), None, strides(*so), None)
    dense = ((1 << 29) * 256, 256, 64)
    assert run(dense, (1 << 40, 1 << 40, 64)) == SHAPE
    assert run(dense, (1 << 40, 1 << 39, 64)) == SHAPE
    assert run((1 << 40, 1 << 40, 64), dense) == SHAPE     # no memory holds such an input either
    assert run((dense[0], dense[1], (1 << 40) + 8), dense) == SHAPE


def test_the_check_of_a_rotary_call_answers_as_the_call_does():
    keep = A.astro_rope_create(64, 64, "halves", (32,))
    p = lambda x: C.c_void_p(x) if x else None  # noqa: E731

    def check(q=0x10000, qo=0x40000, pos=0x30000, B=2, n=8, dtype=0, so=None):
        return A.lib().astro_rope_apply_check(keep.handle, 0, p(q), None, p(pos), 1, B, n, 4, 0, dtype, None, p(qo), None,
                                              None if so is None else C.byref(A.Strides(*so)))

    assert check() == 0 and check(n=0, q=0, qo=0, pos=0) == 0
    assert check(q=0) == 1 and check(B=0) == SHAPE and check(dtype=3) == SHAPE and check(q=0x10002) == 3 and check(so=(0, 256, 64)) == SHAPE
    assert A.lib().astro_rope_apply_check(None, 0, p(1 << 16), None, p(1 << 17), 1, 1, 1, 1, 0, 0, None, p(1 << 18), None, None) == 1
