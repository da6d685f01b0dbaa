"""CPU-side checks of the C ABI of the 8-bit cache, attention over it and sliding-window attention: every refusal comes before
anything is launched, so none of it needs a device; the oracle of 8-bit rows and the gradients that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

from attn_bounds import head
from oracle import cache8 as orc
from paper_2603_17051_b200 import binding as A

P = C.c_void_p(0x10000)
ODD = C.c_void_p(0x10008)
OK, NULL, SHAPE, ALIGN, CAPACITY, UNDERFLOW = 0, 1, 2, 3, 4, 5


def cache(batch=1, heads=2, dim=64, tokens=16, sink=1, window=4, k=0x100000, v=0x900000, held=None, bits=8, nbytes=1 << 20):
    out = C.c_void_p()
    d = A.KVCacheDesc(batch, heads, dim, tokens, sink, window)
    create = A.lib().astro_kvcache8_create if bits == 8 else A.lib().astro_kvcache_create
    assert create(C.byref(d), C.c_void_p(k), C.c_void_p(v), nbytes, C.byref(out)) == OK
    if held:
        s = min(sink, held)
        assert A.lib().astro_kvcache_set_state(out, C.byref(A.KVCacheState(s, 0, held - s, held))) == OK
    return out


def test_storage_and_creation():
    L = A.lib()
    for d, want in (((1, 1, 64, 1, 0, 1), 64 + 16), ((2, 12, 128, 1560, 3, 12), 2 * 12 * 15 * 1560 * 129), ((1, 3, 64, 7, 1, 2), 63 * 64 + 64)):
        assert A.astro_kvcache8_storage_bytes(*d) == want
        desc = A.KVCacheDesc(*d)
        out = C.c_void_p()
        assert L.astro_kvcache8_create(C.byref(desc), P, P, want - 1, C.byref(out)) == CAPACITY
        assert L.astro_kvcache8_create(C.byref(desc), P, P, want, C.byref(out)) == OK and L.astro_kvcache_destroy(out) == OK
        assert L.astro_kvcache8_create(C.byref(desc), ODD, P, want, C.byref(out)) == ALIGN
        assert L.astro_kvcache8_create(C.byref(desc), None, P, want, C.byref(out)) == NULL
    for bad in ((0, 1, 64, 1, 0, 1), (1, 1, 96, 1, 0, 1), (1, 1, 64, 0, 0, 1), (1, 1, 64, 1, -1, 1), (1, 1, 64, 1, 0, 0)):
        assert A.astro_kvcache8_storage_bytes(*bad) == 0
        desc = A.KVCacheDesc(*bad)
        assert L.astro_kvcache8_create(C.byref(desc), P, P, 1 << 30, C.byref(C.c_void_p())) == SHAPE


def test_writing_and_reading_refusals():
    L = A.lib()
    c, wide = cache(held=3), cache(bits=16, held=3)
    append, read = L.astro_kvcache8_append, L.astro_kvcache8_read
    assert append(None, P, P, 1, 0, None, None) == NULL and append(c, None, P, 1, 0, None, None) == NULL and append(c, P, None, 1, 0, None, None) == NULL
    assert append(wide, P, P, 1, 0, None, None) == SHAPE and append(c, P, P, -1, 0, None, None) == SHAPE
    assert append(c, P, P, 1, 3, None, None) == SHAPE and append(c, P, P, 1, -1, None, None) == SHAPE
    assert append(c, ODD, P, 1, 0, None, None) == ALIGN and append(c, P, ODD, 1, 0, None, None) == ALIGN
    assert append(c, P, P, 3, 0, None, None) == CAPACITY and append(c, P, P, 0, 0, None, None) == OK
    for strides, dtype, want in (((0, 128, 60), 0, ALIGN), ((0, 4, 64), 0, ALIGN), ((0, 4, 64), 2, None), ((0, -128, 64), 0, SHAPE),
                                 ((0, 1 << 41, 64), 0, SHAPE)):
        got = append(c, P, P, 1, dtype, C.byref(A.Strides(*strides)), None)
        assert got == want if want is not None else got not in (ALIGN, SHAPE)
    assert read(None, 0, 1, 0, P, P, None) == NULL and read(c, 0, 1, 0, None, P, None) == NULL and read(c, 0, 1, 0, P, None, None) == NULL
    assert read(wide, 0, 1, 0, P, P, None) == SHAPE and read(c, 0, 1, 3, P, P, None) == SHAPE
    for first, count in ((-1, 1), (0, 4), (3, 1), (4, 0), (1, -1), (2, 2147483647)):
        assert read(c, first, count, 0, P, P, None) == SHAPE
    assert read(c, 0, 1, 0, ODD, P, None) == ALIGN and read(c, 3, 0, 0, None, None, None) == OK
    a, b, seen = C.c_int(), C.c_int(), C.c_int64()          # nothing was changed by any of it
    assert L.astro_kvcache_query(c, C.byref(a), C.byref(b), C.byref(seen)) == OK and (a.value, b.value, seen.value) == (1, 2, 3)


def test_calls_that_read_a_16_bit_cache_refuse_an_8_bit_one():
    L = A.lib()
    c, wide, other = cache(held=3), cache(bits=16, held=3, k=0x2000000, v=0x3000000), cache(k=0x4000000, v=0x5000000)
    assert L.astro_chunk_attn_fwd(c, P, P, P, 1, 2, 64, 5, 5, 0.1, P, P, None) == SHAPE
    assert L.astro_chunk_attn_bwd(c, P, P, P, P, P, P, 1, 2, 64, 5, 5, 0.1, P, P, P, P, 1 << 20, None) == SHAPE
    assert L.astro_chunk_attn_bwd_dq(c, P, P, P, P, P, P, 1, 2, 64, 5, 5, 0.1, P, None) == SHAPE
    assert L.astro_chunk_attn_bwd_static(c, P, P, P, P, P, P, 1, 2, 64, 5, 5, 0.1, P, P, P, None) == SHAPE
    assert L.astro_block_pool(c, 0, 1, 16, P, None) == SHAPE
    assert L.astro_block_select(c, P, P, P, 1, 2, 64, 5, 5, 16, 4, 0, P, P, 1 << 20, None) == SHAPE
    assert L.astro_sparse_attn_fwd(c, P, P, P, P, 4, 16, 1, 2, 64, 5, 5, 0.1, P, P, P, 1 << 20, None) == SHAPE
    assert L.astro_sparse_attn_bwd(c, P, P, P, P, 4, 16, P, P, P, 1, 2, 64, 5, 5, 0.1, P, P, P, P, 1 << 20, None) == SHAPE
    assert L.astro_kvcache_fork(c, wide, None, None, -1, None) == SHAPE and L.astro_kvcache_fork(wide, c, None, None, -1, None) == SHAPE
    assert L.astro_kvcache_fork(other, c, None, None, 0, None) == OK                      # an empty fork of two 8-bit caches
    near = cache(k=0x100000 + 5 * 2 * 16 * 64, v=0x900000)
    assert L.astro_kvcache_fork(near, c, None, None, -1, None) == SHAPE                  # storages that overlap by the exponents
    assert L.astro_kvcache_evict(c, 3, None) == UNDERFLOW and L.astro_kvcache_evict(c, 2, None) == OK


@pytest.mark.parametrize("bits", [16, 8])
def test_attention_over_the_cache_refusals(bits):
    L = A.lib()
    c, empty = cache(bits=bits, held=3), cache(bits=bits)
    wrong = bits == 16

    def fwd(cache=c, q=P, k=P, v=P, batch=1, heads=2, dim=64, n_q=100000, n_kc=5, scale=0.1, o=P, lse=P, ws=P, nbytes=1 << 30):
        return L.astro_chunk_attn8_fwd(cache, q, k, v, batch, heads, dim, n_q, n_kc, scale, o, lse, ws, nbytes, None)

    def bwd(cache=c, q=P, k=P, v=P, o=P, lse=P, d_o=P, batch=1, heads=2, dim=64, n_q=100000, n_kc=5, scale=0.1, dq=P, dk=P, dv=P, ws=P, nbytes=1 << 30):
        return L.astro_chunk_attn8_bwd(cache, q, k, v, o, lse, d_o, batch, heads, dim, n_q, n_kc, scale, dq, dk, dv, ws, nbytes, None)

    if wrong:
        assert fwd() == SHAPE and bwd() == SHAPE and L.astro_chunk_attn8_fwd_workspace_bytes(c, 1, 2, 64, 100, 5) == 0
        return
    for f in (fwd, bwd):
        assert f(q=None) == NULL and f(k=None) == NULL and f(v=None) == NULL and f(o=None) == NULL
        for bad in (dict(batch=0), dict(batch=2, cache=cache(batch=3, held=1)), dict(heads=3), dict(dim=128), dict(dim=96), dict(n_q=0),
                    dict(n_kc=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(cache=empty, n_kc=0)):
            assert f(**bad) == SHAPE, bad
        for bad in (dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(o=ODD), dict(ws=ODD), dict(lse=C.c_void_p(0x10002))):
            assert f(**bad) == ALIGN, bad
        assert f(ws=None) == NULL and f(nbytes=100) == CAPACITY
    for bad in ("lse", "d_o", "dq", "dk", "dv"):
        assert bwd(**{bad: None}) == NULL
        assert bad == "lse" or bwd(**{bad: ODD}) == ALIGN
    rows = 2 * 48 * 64 * 2                                       # K or V of the held frames in bf16
    size = L.astro_chunk_attn8_fwd_workspace_bytes
    assert size(c, 1, 2, 64, 100000, 5) == 2 * rows and size(None, 1, 2, 64, 100, 5) == 0
    assert L.astro_chunk_attn8_bwd_workspace_bytes(c, 1, 2, 64, 100, 5) == 2 * rows + 1024
    assert fwd(n_q=100000, nbytes=2 * rows - 1) == CAPACITY and size(c, 1, 2, 64, 0, 5) == 0 and size(c, 1, 2, 65, 100, 5) == 0


def window(fwd=True, q=P, qs=None, k=P, ks=None, v=P, vs=None, lens=None, o=P, lse=P, d_o=P, scale=0.1, dq=P, dk=P, dv=P, ws=P, nbytes=1 << 30,
           desc=True, **d):
    base = dict(batch=2, n_tokens=300, heads=4, kv_heads=2, head_dim=64, block_tokens=1, window_tokens=50, sink_tokens=4)
    base.update(d)
    desc = C.byref(A.WindowDesc(*[base[n] for n, _ in A.WindowDesc._fields_])) if desc else None
    s = [None if x is None else C.byref(A.Strides(*x)) for x in (qs, ks, vs)]
    if fwd:
        return A.lib().astro_window_attn_fwd(desc, q, s[0], k, s[1], v, s[2], lens, scale, o, lse, None)
    return A.lib().astro_window_attn_bwd(desc, q, s[0], k, s[1], v, s[2], lens, o, lse, d_o, scale, dq, dk, dv, ws, nbytes, None)


@pytest.mark.parametrize("fwd", [True, False])
def test_window_refusals(fwd):
    f = lambda **kw: window(fwd, **kw)  # noqa: E731
    assert f(desc=False) == NULL
    for name in ("q", "k", "v", "o") + (() if fwd else ("lse", "d_o", "dq", "dk", "dv", "ws")):
        assert f(**{name: None}) == NULL
        assert name == "lse" or f(**{name: ODD}) == ALIGN
    for bad in (dict(batch=0), dict(n_tokens=-1), dict(n_tokens=(1 << 29) + 1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=96),
                dict(head_dim=256), dict(block_tokens=0), dict(block_tokens=51), dict(window_tokens=0), dict(sink_tokens=-1), dict(batch=65536),
                dict(scale=-0.1), dict(scale=float("inf")), dict(scale=float("nan")), dict(batch=60000, heads=60000, kv_heads=1)):
        assert f(**bad) == SHAPE, bad
    assert f(lens=C.c_void_p(0x10002)) == ALIGN and f(lse=C.c_void_p(0x10002)) == ALIGN
    good = (300 * 4 * 64, 4 * 64, 64)
    for at in ("qs", "ks", "vs"):
        for i, x, want in ((0, 0, SHAPE), (1, 0, SHAPE), (2, 0, SHAPE), (1, -64, SHAPE), (2, 60, ALIGN), (1, 250, ALIGN), (2, 56, SHAPE), (0, 1 << 50, SHAPE)):
            assert f(**{at: good[:i] + (x,) + good[i + 1:]}) == want, (at, i, x)
    assert f(n_tokens=0, q=None, k=None, v=None, o=None, lse=None, d_o=None, dq=None, dk=None, dv=None, ws=None) == OK
    if not fwd:
        need = A.astro_window_attn_bwd_workspace_bytes(2, 4, 300, 64)
        assert need >= 2 * 4 * 300 * 4 and f(nbytes=need - 1) == CAPACITY
        assert A.astro_window_attn_bwd_workspace_bytes(2, 4, 300, 65) == 0 and A.astro_window_attn_bwd_workspace_bytes(0, 4, 300, 64) == 0


def test_tensors_the_binding_refuses():
    q = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        A.astro_window_attn_fwd(q, q, q, 0.1)                    # on the host
    with pytest.raises(ValueError):
        A.astro_chunk_attn8_fwd(None, q, q, q, 0.1)


def test_the_oracle_of_8_bit_rows_is_the_types_own_rounding():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(4000, generator=g, dtype=torch.float64) * torch.exp(3 * torch.randn(4000, generator=g, dtype=torch.float64))
    x = x.clamp(-448, 448).float()
    want = x.to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.e4m3(x.double().numpy()), want)
    rows = torch.randn(50, 64, generator=g, dtype=torch.float64).numpy() * np.exp2(np.arange(-120, 80, 4))[:, None]
    e = orc.exponents(rows)
    top = np.abs(rows).max(-1)
    assert (top <= 448 * np.exp2(e.astype(float))).all() and ((top > 448 * np.exp2(e - 1.0)) | (e == orc.LOWEST_EXP)).all()
    assert (np.abs(orc.stands_for(rows) - rows) <= np.maximum(2.0 ** -4 * np.abs(rows), np.exp2(e - 10.0)[:, None])).all()


def test_the_gradients_that_kernels_are_compared_with_are_the_differences():
    g = torch.Generator().manual_seed(2)
    q, k, v, d_o = (torch.randn(n, 8, generator=g, dtype=torch.float64) for n in (5, 7, 7, 5))
    see = torch.rand(5, 7, generator=g) < 0.6
    see[3] = False                                               # a query that sees nothing
    got = head(q, k, v, 0.3, see, d_o)
    assert not got["o"][0][3].any() and not got["dq"][0][3].any() and got["lse"][0][3] == -torch.inf
    step = 1e-6

    def loss(*x):
        return (head(*x, 0.3, see)["o"][0] * d_o).sum().item()

    for name, i in (("dq", 0), ("dk", 1), ("dv", 2)):
        x = [q, k, v]
        for r in range(len(x[i])):
            for c in range(8):
                up, down = [t.clone() for t in x], [t.clone() for t in x]
                up[i][r, c] += step
                down[i][r, c] -= step
                assert abs((loss(*up) - loss(*down)) / (2 * step) - got[name][0][r, c].item()) < 1e-7
