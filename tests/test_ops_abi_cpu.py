"""CPU-side checks of the C ABI of rotary positions, key blocks, attention over lists and cache forks: every refusal comes
before anything is launched, so none of it needs a device; tables and counts are host arithmetic."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import rope as rope_orc
from oracle import sparse_attn as orc
from paper_2603_17051_b200 import binding as A

P = C.c_void_p(0x10000)
NULL, SHAPE, ALIGN, CAPACITY = 1, 2, 3, 4


def cache(batch=1, heads=2, dim=64, tokens=16, sink=1, window=4, k=0x100000, v=0x900000, held=None):
    out = C.c_void_p()
    d = A.KVCacheDesc(batch, heads, dim, tokens, sink, window)
    assert A.lib().astro_kvcache_create(C.byref(d), C.c_void_p(k), C.c_void_p(v), 1 << 20, C.byref(out)) == 0
    if held:
        s = min(sink, held)
        assert A.lib().astro_kvcache_set_state(out, C.byref(A.KVCacheState(s, 0, held - s, held))) == 0
    return out


# ------------------------------------------------------------------------------------------------ rotary positions

def desc(**kw):
    base = dict(head_dim=64, rot_dim=64, layout=0, axes=1, axis_pairs=(32,), base=10000.0, scaling=0, scaled_axes=1, factor=1.0,
                original_length=4096.0, ramp_low=1.0, ramp_high=32.0, magnitude=0.0)
    base.update(kw)
    base["axis_pairs"] = (C.c_int * 4)(*base["axis_pairs"])
    return A.RopeDesc(*[base[n] for n, _ in A.RopeDesc._fields_])


@pytest.mark.parametrize("bad", [dict(head_dim=4), dict(head_dim=60), dict(head_dim=264), dict(rot_dim=63, axis_pairs=(31,)), dict(rot_dim=0),
                                 dict(rot_dim=66, axis_pairs=(33,)), dict(layout=2), dict(layout=-1), dict(axes=0), dict(axes=5),
                                 dict(axis_pairs=(31,)), dict(axes=2, axis_pairs=(33, -1)), dict(base=0.0), dict(base=float("nan")),
                                 dict(base=float("inf")), dict(scaling=4), dict(scaling=1, factor=0.5), dict(scaling=2, factor=float("nan")),
                                 dict(scaling=3, original_length=0.0), dict(scaling=3, ramp_low=2.0, ramp_high=2.0),
                                 dict(magnitude=-1.0), dict(magnitude=float("inf"))])
def test_rope_descriptors_that_are_refused(bad):
    out = C.c_void_p()
    assert A.lib().astro_rope_create(C.byref(desc(**bad)), C.byref(out)) == SHAPE and not out.value


def test_rope_table_and_null_arguments():
    L = A.lib()
    assert L.astro_rope_create(None, C.byref(C.c_void_p())) == NULL and L.astro_rope_create(C.byref(desc()), None) == NULL
    assert L.astro_rope_destroy(None) == NULL and L.astro_rope_frequencies(None, None, None) == NULL
    for scaling, factor, cut, axes in (("none", 1.0, (32,), None), ("linear", 3.0, (10, 11, 11), (1,)), ("base", 8.0, (1, 31), None),
                                       ("ramp", 16.0, (20, 12), None), ("ramp", 16.0, (20, 12), (0,))):
        rope = A.astro_rope_create(64, 64, "halves", cut, base=5000.0, scaling=scaling, factor=factor, scaled_axes=axes, original_length=777)
        f, _ = rope_orc.frequencies(cut, 5000.0, scaling, factor, axes, 777)
        got, size = A.astro_rope_frequencies(rope)
        assert np.allclose(got, f, rtol=1e-13, atol=0) and size == pytest.approx(rope_orc.magnitude(scaling, factor), abs=1e-15)
    rope = A.astro_rope_create(64, 32, "halves", (16,), magnitude=0.25)
    assert A.astro_rope_frequencies(rope)[1] == 0.25
    with pytest.raises(A.AstroError):
        A.astro_rope_create(64, 10, "halves", (1, 1, 1, 1, 1))
    with pytest.raises(KeyError):
        A.astro_rope_create(64, 64, "sideways", (32,))


def test_rope_apply_arguments():
    L = A.lib()
    r = A.astro_rope_create(64, 64, "halves", (32,)).handle
    keep = A.astro_rope_create(64, 64, "halves", (32,))
    r = keep.handle

    def run(rope=r, inv=0, q=0x10000, k=0x20000, pos=0x30000, pb=1, B=2, n=8, hq=4, hk=4, dtype=0, si=None, qo=0x40000, ko=0x50000, so=None):
        v = lambda x: C.c_void_p(x) if x else None  # noqa: E731
        s = lambda x: None if x is None else C.byref(A.Strides(*x))  # noqa: E731
        return L.astro_rope_apply(rope, inv, v(q), v(k), v(pos), pb, B, n, hq, hk, dtype, s(si), v(qo), v(ko), s(so), None)

    assert run(rope=None) == NULL and run(q=0) == NULL and run(qo=0) == NULL and run(pos=0) == NULL
    assert run(ko=0) == NULL and run(k=0) == NULL                          # k and k_out come together
    assert run(B=0) == SHAPE and run(n=-1) == SHAPE and run(hq=0) == SHAPE and run(hk=0) == SHAPE and run(pb=3) == SHAPE
    assert run(dtype=3) == SHAPE and run(inv=2) == SHAPE and run(B=1 << 20, n=1 << 12, pb=1) == SHAPE
    assert run(n=0) == 0 and run(n=0, q=0, qo=0, pos=0) == 0                # an empty call
    assert run(q=0x10002) == ALIGN and run(ko=0x50008) == ALIGN and run(pos=0x30002) == ALIGN
    dense = (8 * 4 * 64, 4 * 64, 64)
    assert run(si=(8 * 4 * 64, 4 * 64 + 4, 64)) == ALIGN                    # 8 bytes off in bf16 ...
    assert run(so=(8 * 4 * 64 + 4, 4 * 64, 64)) == ALIGN
    assert run(si=(-dense[0], dense[1], dense[2])) == SHAPE and run(so=(dense[0], dense[1], -64)) == SHAPE
    for overlap in ((0, 256, 64), (dense[0], 0, 64), (dense[0], 256, 0), (dense[0], 256, 56), (dense[0] - 256, 256, 64), (64, 256, 64)):
        assert run(so=overlap) == SHAPE, overlap
    assert run(hk=2) == SHAPE                                               # contiguous tensors of other head counts: two calls
    assert run(qo=0x50000) == SHAPE and run(qo=0x20000) == SHAPE and run(ko=0x10000) == SHAPE
    assert run(qo=0x10000, ko=0x20000, so=(dense[0] * 2, dense[1], dense[2])) == SHAPE   # in place needs equal strides


# ------------------------------------------------------------------------------------------------ key blocks

def test_block_counts_follow_the_oracle():
    for tokens, sink, window, held in ((16, 1, 4, 3), (7, 0, 3, 2), (121, 2, 2, 0)):
        h = cache(tokens=tokens, sink=sink, window=window, held=held)
        a, b = C.c_int(), C.c_int()
        for block in range(8, 129, 8):
            for n_kc in (0, 1, block, 3 * block + 1):
                assert A.lib().astro_block_count(h, n_kc, block, C.byref(a), C.byref(b)) == 0
                ranges = orc.key_blocks(held, tokens, n_kc, block)
                assert a.value + b.value == len(ranges)
                assert b.value == sum(first >= held * tokens for first, _ in ranges)
        for block in (0, -8, 4, 12, 136):
            assert A.lib().astro_block_count(h, 5, block, C.byref(a), C.byref(b)) == SHAPE
        assert A.lib().astro_block_count(h, -1, 64, None, None) == SHAPE
        A.lib().astro_kvcache_destroy(h)
    assert A.astro_block_count(None, 100, 64) == (0, 2)


def test_pool_and_select_arguments():
    L = A.lib()
    h = cache(held=4)
    pool = lambda c=h, first=0, n=1, block=16, out=P: L.astro_block_pool(c, first, n, block, out, None)  # noqa: E731
    assert pool(c=None) == NULL and pool(out=None) == NULL and pool(out=C.c_void_p(0x10008)) == ALIGN
    assert pool(block=20) == SHAPE and pool(first=-1) == SHAPE and pool(n=-1) == SHAPE and pool(first=2, n=3) == SHAPE and pool(first=5, n=0) == SHAPE
    assert pool(first=4, n=0) == 0
    need = L.astro_block_select_workspace_bytes(1, 2, 64, 200, 40, 16)
    assert need == 2 * 64 * 4 * (2 + 3)
    for bad in ((0, 2, 64, 1, 0, 16), (1, 0, 64, 1, 0, 16), (1, 2, 80, 1, 0, 16), (1, 2, 64, 0, 0, 16), (1, 2, 64, 1, -1, 16), (1, 2, 64, 1, 0, 15)):
        assert L.astro_block_select_workspace_bytes(*bad) == 0

    def select(c=h, pooled=P, q=P, k=P, B=1, H=2, D=64, n_q=200, n_kc=40, block=16, n=4, keep=0, out=P, ws=P, size=need):
        return L.astro_block_select(c, pooled, q, k, B, H, D, n_q, n_kc, block, n, keep, out, ws, size, None)

    assert select(q=None) == NULL and select(k=None) == NULL and select(out=None) == NULL and select(ws=None) == NULL
    assert select(pooled=None) == NULL                                      # the cache holds frames
    assert select(H=3) == SHAPE and select(D=128) == SHAPE and select(D=96) == SHAPE and select(B=0) == SHAPE and select(n_q=0) == SHAPE
    assert select(block=9) == SHAPE and select(n=0) == SHAPE and select(n=65537) == SHAPE and select(keep=4) == SHAPE and select(keep=-1) == SHAPE
    assert select(c=None, pooled=None, n_kc=0) == SHAPE                     # no key at all
    assert select(c=None, pooled=None, n_kc=24577 * 8, block=8, size=1 << 40) == SHAPE
    assert select(q=C.c_void_p(0x10002)) == ALIGN and select(ws=C.c_void_p(0x10008)) == ALIGN and select(out=C.c_void_p(0x10002)) == ALIGN
    assert select(size=need - 1) == CAPACITY
    L.astro_kvcache_destroy(h)


def test_sparse_attention_arguments():
    L = A.lib()
    h = cache(held=4)

    def fwd(c=h, q=P, k=P, v=P, blocks=P, n=4, block=16, B=1, H=2, D=64, n_q=300, n_kc=40, scale=0.1, o=P, lse=P, ws=None, size=0):
        return L.astro_sparse_attn_fwd(c, q, k, v, blocks, n, block, B, H, D, n_q, n_kc, scale, o, lse, ws, size, None)

    assert fwd(q=None) == NULL and fwd(o=None) == NULL and fwd(blocks=None) == NULL and fwd(k=None) == NULL and fwd(v=None) == NULL
    for bad in (dict(n=0), dict(n=65537), dict(block=7), dict(block=136), dict(B=0), dict(H=3), dict(D=96), dict(n_q=0), dict(n_kc=-1),
                dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(c=None, n_kc=0), dict(B=65536)):
        assert fwd(**bad) == SHAPE, bad
    assert fwd(q=C.c_void_p(0x10008)) == ALIGN and fwd(lse=C.c_void_p(0x10002)) == ALIGN and fwd(blocks=C.c_void_p(0x10001)) == ALIGN
    # scratch: none for many queries, for short lists and for one or two queries; parts for a few queries with long lists
    size = L.astro_sparse_attn_fwd_workspace_bytes
    assert size(1, 12, 128, 4680, 64, 120) == 0 and size(1, 2, 64, 5, 11, 128) == 0 and size(1, 2, 64, 2, 64, 128) == 0
    need = size(1, 2, 64, 5, 64, 128)
    assert need > 0 and need % (2 * 5 * 65 * 4) == 0
    long = dict(n_q=5, n=64, block=128)
    assert fwd(**long) == NULL and fwd(**long, ws=P, size=need - 1) == CAPACITY and fwd(**long, ws=C.c_void_p(0x10004), size=need) == ALIGN
    for bad in ((0, 2, 64, 1, 1, 64), (1, 2, 64, 0, 1, 64), (1, 2, 64, 1, 0, 64), (1, 2, 65, 1, 1, 64), (1, 2, 64, 1, 1, 63)):
        assert size(*bad) == 0

    def bwd(c=h, q=P, k=P, v=P, blocks=P, n=4, block=16, o=P, lse=P, d_o=P, B=1, H=2, D=64, n_q=300, n_kc=40, scale=0.1, dq=P, dk=P, dv=P,
            ws=P, size=1 << 30):
        return L.astro_sparse_attn_bwd(c, q, k, v, blocks, n, block, o, lse, d_o, B, H, D, n_q, n_kc, scale, dq, dk, dv, ws, size, None)

    for name in ("q", "k", "v", "blocks", "o", "lse", "d_o", "dq", "dk", "dv", "ws"):
        assert bwd(**{name: None}) == NULL, name
        assert bwd(**{name: C.c_void_p(0x10002)}) == ALIGN, name
    for bad in (dict(n=0), dict(n=65537), dict(block=12), dict(H=3), dict(n_q=0), dict(scale=-0.5), dict(c=None, n_kc=0), dict(n_q=128 * 32768, n=65536)):
        assert bwd(**bad) == SHAPE, bad
    need = L.astro_sparse_attn_bwd_workspace_bytes(1, 2, 64, 300, 40, 4, 16)
    assert need == (2 * 300 * 4 + 255) // 256 * 256 + 2 * 3 * 3 * 4 and bwd(size=need - 1) == CAPACITY
    assert L.astro_sparse_attn_bwd_workspace_bytes(1, 2, 64, 300, -1, 4, 16) == 0
    L.astro_kvcache_destroy(h)


# ------------------------------------------------------------------------------------------------ forks

def test_fork_arguments_and_the_state_of_an_empty_fork():
    L = A.lib()
    src = cache(batch=2, held=4)
    one = cache(batch=1, held=3)
    make = lambda **kw: cache(**{**dict(batch=2, k=0x2000000, v=0x2900000, held=2), **kw})  # noqa: E731
    arr = lambda *f: (C.c_int * max(1, len(f)))(*f)  # noqa: E731
    dst = make()
    run = lambda d=dst, s=src, parents=None, frames=None, n=-1: L.astro_kvcache_fork(d, s, parents, frames, n, None)  # noqa: E731
    assert run(d=None) == NULL and run(s=None) == NULL and run(n=2) == NULL
    assert run(n=-2) == SHAPE and run(frames=arr(0), n=-1) == SHAPE
    assert run(s=dst) == SHAPE                                              # onto itself
    for other in (make(heads=1), make(dim=128), make(tokens=8), make(batch=3)):
        assert run(d=other) == SHAPE
        L.astro_kvcache_destroy(other)
    size = 2 * 2 * 5 * 16 * 64 * 2                                          # bytes of one storage tensor
    for k, v in ((0x100000 + size - 16, 0x2900000), (0x2000000, 0x900000 - size + 16), (0x900000, 0x2900000)):
        other = make(k=k, v=v)
        assert run(d=other) == SHAPE                                        # storage that overlaps the source's
        L.astro_kvcache_destroy(other)
    assert run(frames=arr(4), n=1) == SHAPE and run(frames=arr(-1), n=1) == SHAPE
    assert run(frames=arr(0, 1, 2, 3, 0, 1), n=6) == CAPACITY
    assert run(parents=C.c_void_p(0x30002)) == ALIGN
    s = A.KVCacheState()
    L.astro_kvcache_get_state(dst, C.byref(s))
    assert (s.sink_held, s.window_held, s.frames_seen) == (1, 1, 2)         # every refusal left it alone
    assert run(n=0) == 0 and run(s=one, frames=arr(), n=0) == 0             # nothing to copy: the destination is emptied
    L.astro_kvcache_get_state(dst, C.byref(s))
    assert (s.sink_held, s.window_head, s.window_held, s.frames_seen) == (0, 0, 0, 3)
    for h in (src, one, dst):
        L.astro_kvcache_destroy(h)
