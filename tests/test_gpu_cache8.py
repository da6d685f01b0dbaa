"""The cache in 8 bits on the GPU: what is written against the fp64 oracle, bit for bit."""
import numpy as np
import pytest

from oracle import cache8 as orc

pytestmark = pytest.mark.gpu


def modules():
    import torch
    from paper_2603_17051_b200 import binding as A
    return torch, A


def rows(torch, shape, dtype, seed):
    """Rows of very different sizes, zeros among them, elements of very different sizes within a row."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda") * torch.exp(torch.randn(shape, generator=g, device="cuda"))
    power = torch.randint(-14 if dtype is torch.float16 else -130, 8 if dtype is torch.float16 else 110, shape[:-1], generator=g, device="cuda")
    usual = torch.rand(shape[:-1], generator=g, device="cuda") < 0.7
    x = x.double() * torch.where(usual, 1.0, torch.exp2(power.double()))[..., None]
    x[torch.rand(shape[:-1], generator=g, device="cuda") < 0.05] = 0.0
    return x.to(dtype)


def want(x):
    return orc.stands_for(x.double().cpu().numpy())


def same(got, ref):
    return np.array_equal(got.double().cpu().numpy(), ref, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("B,H,D,T,S,L,frames", [(1, 1, 64, 1, 0, 1, 1), (2, 3, 128, 7, 1, 4, 3), (1, 12, 128, 33, 3, 12, 2), (3, 1, 64, 250, 0, 2, 1),
                                                (1, 5, 64, 1, 4, 300, 289), (1, 40, 128, 16, 2, 3, 4)])
def test_written_and_read_back(dtype, B, H, D, T, S, L, frames):
    torch, A = modules()
    kind = getattr(torch, dtype)
    cache = A.astro_kvcache8_create(B, H, D, T, S, L)
    k, v = (rows(torch, (B, frames * T, H, D), kind, seed) for seed in (1, 2))
    A.astro_kvcache8_append(cache, k, v, frames)
    for out in (torch.bfloat16, torch.float32):           # both hold every value exactly
        a, b = A.astro_kvcache8_read(cache, dtype=out)
        assert a.dtype is out and same(a, want(k)) and same(b, want(v))
    half, _ = A.astro_kvcache8_read(cache, dtype=torch.float16)
    assert torch.equal(half, torch.from_numpy(want(k)).to(torch.float16).cuda())     # one rounding; infinite beyond its range
    if kind is torch.bfloat16:
        a, b = A.astro_kvcache_export(cache)
        assert same(a, want(k)) and same(b, want(v))


def test_against_the_type_itself():
    """The oracle's rounding is e4m3's: every bf16 number between 0 and 448 beside a row's largest."""
    torch, A = modules()
    x = torch.arange(0, 1 << 15, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = x[x.isfinite() & (x <= 448)]
    x = x[:len(x) // 63 * 63].view(1, -1, 1, 63)
    x = torch.cat([x, torch.full_like(x[..., :1], 448.0)], -1).contiguous()          # e = 0
    cache = A.astro_kvcache8_create(1, 1, 64, x.shape[1], 0, 1)
    A.astro_kvcache8_append(cache, x, -x, 1)
    k, v = A.astro_kvcache8_read(cache)
    ref = x.float().to(torch.float8_e4m3fn).float()
    assert torch.equal(k.float(), ref) and torch.equal(v.float(), -ref)


def test_infinities_nan_and_the_ends_of_the_range():
    torch, A = modules()
    D = 64
    x = torch.ones(1, 8, 1, D)
    x[0, 0, 0, 3], x[0, 0, 0, 5], x[0, 0, 0, 7] = float("inf"), float("-inf"), float("nan")
    x[0, 1] = float("nan")
    x[0, 2] = 3.3895313892515355e38                                                   # bf16's largest
    x[0, 3] = 2.0 ** -133                                                             # bf16's smallest
    x[0, 4], x[0, 4, 0, 0] = 2.0 ** -120, 448.0
    x[0, 5] = -0.0
    x[0, 6], x[0, 6, 0, 1] = 1.75 * 2.0 ** -116, -1.75 * 2.0 ** -125
    x = x.bfloat16().cuda()
    cache = A.astro_kvcache8_create(1, 1, D, 8, 0, 1)
    A.astro_kvcache8_append(cache, x, x, 1)
    k, _ = A.astro_kvcache8_read(cache)
    assert same(k, want(x))
    got = k[0, 0, 0]
    assert got[[3, 5, 7]].isnan().all() and (got[[0, 1, 2, 4, 6]] == 1).all()


def test_ring_strides_ranges_and_what_stays_untouched():
    torch, A = modules()
    B, H, D, T, S, L = 2, 3, 128, 5, 2, 4
    nbytes = A.astro_kvcache8_storage_bytes(B, H, D, T, S, L)
    assert nbytes == B * H * (S + L) * T * D + (B * H * (S + L) * T + 15) // 16 * 16
    stores = [torch.full((nbytes + 64,), 77, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = A.astro_kvcache8_create(B, H, D, T, S, L, k_storage=stores[0][:nbytes], v_storage=stores[1][:nbytes])
    packed = rows(torch, (B, 12 * T, 3, H, D), torch.bfloat16, 5)                     # q, k and v beside each other
    model = []

    def put(first, count):
        part = packed[:, first * T:(first + count) * T]
        A.astro_kvcache8_append(cache, part[:, :, 1], part[:, :, 2], count)
        model.extend(range(first, first + count))

    put(0, 4)
    free = (S + 2) * T                                                                # slots 4 and 5 of every head were not written
    codes = stores[0][:B * H * (S + L) * T * D].view(B, H, (S + L) * T, D)
    assert (codes[:, :, free:] == 77).all() and all((s[nbytes:] == 77).all() for s in stores)
    put(4, 2)
    A.astro_kvcache_evict(cache, 3); del model[S:S + 3]
    put(6, 2)                                                                         # slots in two pieces of the ring
    A.astro_kvcache_evict(cache, 1); del model[S:S + 1]
    put(8, 2)
    held = len(model)
    assert A.astro_kvcache_query(cache)[:2] == (S, held - S)
    at = torch.cat([torch.arange(f * T, (f + 1) * T) for f in model])
    ref = [want(packed[:, at, i]) for i in (1, 2)]
    for first in range(held + 1):
        for count in range(held - first + 1):
            got = A.astro_kvcache8_read(cache, first, count)
            assert all(same(a, r[:, first * T:(first + count) * T]) for a, r in zip(got, ref))
    with pytest.raises(A.AstroError):
        A.astro_kvcache8_append(cache, packed[:, :T, 1], packed[:, :T, 2], 1)        # full
    state = A.astro_kvcache_get_state(cache)                                          # the bytes and the record are the cache
    other = A.astro_kvcache8_create(B, H, D, T, S, L, k_storage=stores[0].clone(), v_storage=stores[1].clone())
    A.astro_kvcache_set_state(other, state)
    assert all(same(a, r) for a, r in zip(A.astro_kvcache8_read(other), ref))
    A.astro_kvcache_reset(cache)
    assert A.astro_kvcache8_read(cache)[0].shape[1] == 0


def test_offsets_beyond_32_bits():
    """Storage of more than 4 GiB: the last slot's rows."""
    torch, A = modules()
    H, D, T, L = 8, 128, 4096, 1100                                                    # 4.6 GB each
    cache = A.astro_kvcache8_create(1, H, D, T, 0, L)
    A.astro_kvcache_set_state(cache, A.KVCacheState(0, L - 1, 0, 0))
    k, v = (rows(torch, (1, 2 * T, H, D), torch.bfloat16, s) for s in (8, 9))
    A.astro_kvcache_set_state(cache, A.KVCacheState(0, L - 1, 1, 1))
    A.astro_kvcache8_append(cache, k[:, T:].contiguous(), v[:, T:].contiguous(), 1)   # into slot 0
    A.astro_kvcache_evict(cache, 2)
    A.astro_kvcache_set_state(cache, A.KVCacheState(0, L - 2, 1, 1))
    A.astro_kvcache8_append(cache, k[:, :T].contiguous(), v[:, :T].contiguous(), 1)   # into slot L - 1
    A.astro_kvcache_set_state(cache, A.KVCacheState(0, L - 1, 2, 2))
    got = A.astro_kvcache8_read(cache)
    assert same(got[0], want(k)) and same(got[1], want(v))
    A.astro_last_device_status()


def test_forks_copy_rows_as_they_are():
    torch, A = modules()
    H, D, T = 3, 64, 7
    src = A.astro_kvcache8_create(2, H, D, T, 1, 5)
    k, v = (rows(torch, (2, 5 * T, H, D), torch.bfloat16, s) for s in (3, 4))
    A.astro_kvcache8_append(src, k, v, 5)
    dst = A.astro_kvcache8_create(4, H, D, T, 2, 40)
    parents = torch.tensor([1, 0, 7, 1], dtype=torch.int32, device="cuda")
    frames = [3, 0, 4] + [2] * 36                                # more than one launch takes
    A.astro_kvcache_fork(dst, src, parents=parents, frames=frames)
    at = torch.cat([torch.arange(f * T, (f + 1) * T) for f in frames])
    for got, x in zip(A.astro_kvcache8_read(dst, dtype=torch.float32), (k, v)):
        ref = want(x[:, at])
        assert same(got[[0, 1, 3]], ref[[1, 0, 1]]) and not got[2].any()
