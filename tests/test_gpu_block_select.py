"""GPU parity of the block means and of the choice of key blocks against the fp64 oracle."""
import numpy as np
import pytest

from helpers import dev_bf16, f64
from oracle import sparse_attn as orc
from oracle.rolling_attn import bf16_bits_to_f64
from paper_2603_17051_b200 import synth

pytestmark = pytest.mark.gpu


def ring(A, Bc, H, D, T, S, L, evicted, held, seed, poison=False):
    """A cache whose window has wrapped: `evicted` window frames gone, `held` frames left; and its keys in logical order."""
    import torch
    cache = A.astro_kvcache_create(Bc, H, D, T, S, L)
    if poison:
        cache.k_storage.fill_(0xff)          # NaN in every slot that is never written
        cache.v_storage.fill_(0xff)
    kept_k, kept_v = [], []
    sink = 0
    for f in range(held + evicted):
        kb, vb = (synth.normal_bf16(seed + 2 * f + i, (Bc, T, H, D)) for i in range(2))
        if len(kept_k) - sink == L or (sink == S and evicted > 0 and len(kept_k) > sink):
            A.astro_kvcache_evict(cache, 1)
            del kept_k[sink], kept_v[sink]
            evicted -= 1
        A.astro_kvcache_append(cache, dev_bf16(kb), dev_bf16(vb), 1)
        kept_k.append(bf16_bits_to_f64(kb)); kept_v.append(bf16_bits_to_f64(vb))
        if sink < S:
            sink += 1
    cat = lambda x: np.concatenate(x, 1) if x else np.zeros((Bc, 0, H, D))  # noqa: E731
    return cache, cat(kept_k), cat(kept_v), len(kept_k)


CASES = [  # Bc, B, H, D, T, S, L, evicted, held, n_q, n_kc, block, n_select
    (1, 1, 2, 64, 16, 0, 6, 0, 3, 48, 48, 16, 5),
    (1, 3, 1, 128, 100, 1, 4, 3, 5, 300, 130, 64, 7),
    (2, 2, 2, 128, 121, 2, 3, 2, 4, 1, 1, 120, 4),
    (1, 1, 1, 64, 7, 0, 9, 4, 6, 700, 0, 8, 3),
    (1, 2, 2, 64, 40, 3, 2, 0, 2, 5, 1000, 24, 64),
    (1, 1, 1, 128, 33, 0, 3, 0, 0, 129, 500, 128, 2),
]


@pytest.mark.parametrize("Bc,B,H,D,T,S,L,evicted,held,n_q,n_kc,block,n_select", CASES)
@pytest.mark.parametrize("keep", [0, 1, 2, 3])
def test_choice_matches_the_oracle(Bc, B, H, D, T, S, L, evicted, held, n_q, n_kc, block, n_select, keep):
    from paper_2603_17051_b200 import binding as A
    cache, kx, _, frames = ring(A, Bc, H, D, T, S, L, evicted, held, 500)
    sink, win, _ = A.astro_kvcache_query(cache)
    assert sink + win == frames
    qb, kb = synth.normal_bf16(900, (B, n_q, H, D)), synth.normal_bf16(901, (B, max(1, n_kc), H, D))
    kc = dev_bf16(kb) if n_kc else None
    pooled = A.astro_block_pool(cache, block)
    got = A.astro_block_select(cache, pooled, dev_bf16(qb), kc, block, n_select, keep=keep).cpu().numpy()
    ranges = orc.key_blocks(frames, T, n_kc, block)
    per = -(-T // block)
    assert A.astro_block_count(cache, n_kc, block) == (frames * per, -(-n_kc // block))
    kept = (set(range(sink * per)) if keep & 1 else set()) | (set(range(frames * per, len(ranges))) if keep & 2 else set())
    q, k = bf16_bits_to_f64(qb), bf16_bits_to_f64(kb)[:, :n_kc]
    for b in range(B):
        for h in range(H):
            keys = np.concatenate([kx[b if Bc > 1 else 0, :, h], k[b, :, h]])
            want = orc.select(q[b, :, h], keys, ranges, n_select, kept)
            assert np.array_equal(got[b, h], want), (b, h)


def test_means_of_new_frames_only_and_their_slots():
    import torch
    from paper_2603_17051_b200 import binding as A
    cache, kx, _, frames = ring(A, 2, 3, 64, 50, 1, 4, 5, 5, 40)
    whole = A.astro_block_pool(cache, 16)
    assert whole.shape == (2, 3, 5, 4, 64)
    part = torch.full_like(whole, 7.0)
    A.astro_block_pool(cache, 16, first_frame=frames - 2, n_frames=2, pooled=part)
    changed = (part != 7.0).flatten(3).any(-1)[0, 0]
    assert changed.sum() == 2 and torch.equal(part[:, :, changed], whole[:, :, changed])
    A.astro_block_pool(cache, 16, first_frame=1, n_frames=0, pooled=part)
    # every block's mean, found by its frame's storage slot: fp32 rounding of an fp64 sum, half a step
    st = A.astro_kvcache_get_state(cache)
    slots = list(range(st.sink_held)) + [1 + (st.window_head + i) % 4 for i in range(st.window_held)]
    got = f64(whole)
    for f, slot in enumerate(slots):
        for i, (a, b) in enumerate(orc.key_blocks(1, 50, 0, 16)):
            want = kx[:, f * 50 + a:f * 50 + b].mean(1)
            assert (np.abs(got[:, :, slot, i] - want) <= 2.0 ** -24 * np.abs(want) + 1e-16).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("block", [8, 24, 120])
def test_means_of_values_far_apart_and_beyond_fp32(D, block):
    """Sums in fp64 whatever the exponents: neighbours 2^80 apart, terms that cancel, a sum beyond fp32's range, denormals,
    negative zeros, infinities and NaN."""
    import math
    import torch
    from paper_2603_17051_b200 import binding as A
    T = 121
    g = np.random.default_rng(block + D)
    x = torch.from_numpy(np.ldexp(g.standard_normal((1, T, 2, D)), g.integers(-40, 41, (1, T, 2, D)))).bfloat16()
    x[:, 1::2, :, 1] = -x[:, 0:-1:2, :, 1]                     # every pair cancels
    x[:, :, :, 2] = torch.finfo(torch.bfloat16).max            # two of them overflow fp32, their mean does not
    x[:, :, :, 3] = 2.0 ** -133                                # the smallest denormal
    x[:, :, :, 4] = -0.0
    x[:, 5, :, 5] = float("inf")
    x[:, 2, :, 6], x[:, 3, :, 6] = float("inf"), float("-inf")
    x[:, 7, :, 7] = float("nan")
    cache = A.astro_kvcache_create(1, 2, D, T, 0, 1)
    A.astro_kvcache_append(cache, x.cuda(), x.cuda(), 1)
    got = f64(A.astro_block_pool(cache, block))[0, :, 0]
    want_all = x.double().numpy()[0]
    for h in range(2):
        for i, a in enumerate(range(0, T, block)):
            rows = want_all[a:a + block, h]
            for d in range(D):
                col = rows[:, d]
                if not np.isfinite(col).all():
                    want = col.sum()
                    assert np.isnan(got[h, i, d]) if np.isnan(want) else got[h, i, d] == want, (h, i, d)
                    continue
                want = math.fsum(col) / len(col)
                # each addition in fp64, the product with the rounded inverse, one rounding to fp32 (denormals: 2^-150)
                bound = (len(col) + 2) * 2.0 ** -53 * math.fsum(np.abs(col)) / len(col) + 2.0 ** -24 * abs(want) + 2.0 ** -150
                assert abs(got[h, i, d] - want) <= bound * (1 + 1e-6), (h, i, d, got[h, i, d], want)


def test_ties_take_the_lower_block_and_nan_comes_last():
    import torch
    from paper_2603_17051_b200 import binding as A
    H, D, block, n = 1, 64, 8, 9
    k = torch.ones((1, n * block, H, D), dtype=torch.bfloat16, device="cuda")
    q = torch.ones((1, 3, H, D), dtype=torch.bfloat16, device="cuda")
    k[:, 2 * block:3 * block] = 2.0                       # one clear winner
    k[:, 0:1] = float("nan")                              # block 0 has no number for a mean
    k[:, 4 * block] = float("inf")                        # block 4 scores infinity
    k[:, 5 * block] = float("-inf")                       # block 5 minus infinity: still before NaN
    sel = lambda m, **kw: A.astro_block_select(None, None, q, k, block, m, **kw)[0, 0, 0].tolist()  # noqa: E731
    assert sel(2) == [2, 4] and sel(4) == [1, 2, 3, 4] and sel(7) == [1, 2, 3, 4, 6, 7, 8]
    assert sel(8) == [1, 2, 3, 4, 5, 6, 7, 8] and sel(9) == list(range(9)) and sel(11) == list(range(9)) + [-1, -1]
    assert sel(3, keep=A.KEEP_CHUNK) == [0, 1, 2]         # kept blocks are equal among themselves
    z = torch.zeros_like(q)
    z[:, :, :, 0] = -0.0
    k2 = torch.randn_like(k.float()).bfloat16()
    assert A.astro_block_select(None, None, z, k2, block, 4)[0, 0, 0].tolist() == [0, 1, 2, 3]   # every score is zero


def test_many_blocks_and_the_limit():
    import torch
    from paper_2603_17051_b200 import binding as A
    D, block = 64, 8
    for n_blocks in (6145, 24576):
        k = torch.randn(1, n_blocks * block, 1, D, device="cuda").bfloat16()
        q = torch.randn(1, 200, 1, D, device="cuda").bfloat16()
        got = A.astro_block_select(None, None, q, k, block, 100).cpu().numpy()[0, 0]
        ranges = orc.key_blocks(0, 1, n_blocks * block, block)
        assert np.array_equal(got, orc.select(f64(q)[0, :, 0], f64(k)[0, :, 0], ranges, 100))
    with pytest.raises(A.AstroError) as e:
        A.astro_block_select(None, None, q, torch.zeros(1, 24577 * block, 1, D, device="cuda").bfloat16(), block, 4)
    assert e.value.status == 2


def test_refusals():
    import torch
    from paper_2603_17051_b200 import binding as A
    q = torch.zeros(1, 4, 2, 64, device="cuda").bfloat16()
    k = torch.zeros(1, 40, 2, 64, device="cuda").bfloat16()
    for block in (0, 12, 136):
        with pytest.raises(A.AstroError) as e:
            A.astro_block_select(None, None, q, k, block, 4, workspace=torch.empty(4096, dtype=torch.uint8, device="cuda"))
        assert e.value.status == 2
    for bad, status in ((dict(n_select=0), 2), (dict(keep=4), 2), (dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), 4)):
        kw = dict(n_select=4)
        kw.update(bad)
        with pytest.raises(A.AstroError) as e:
            A.astro_block_select(None, None, q, k, 8, **kw)
        assert e.value.status == status
    with pytest.raises(A.AstroError) as e:                # no key at all
        A.astro_block_select(None, None, q, None, 8, 4)
    assert e.value.status == 2
    for args in ((q.float(), k), (q, k.cpu()), (q, k[:, :, :1].contiguous())):
        with pytest.raises(ValueError):
            A.astro_block_select(None, None, *args, 8, 4)
