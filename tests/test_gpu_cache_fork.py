"""Forking a cache: bit-exact copies of chosen frames for chosen parents, and attention over the result."""
import numpy as np
import pytest

from helpers import dev_bf16, host_bits
from paper_2603_17051_b200 import synth
from test_gpu_block_select import ring

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("src_b,dst_b,parents,frames", [(1, 3, None, None), (2, 2, None, [4, 0, 0, 2]), (3, 5, [2, 2, 0, 1, 2], [1, 3]),
                                                        (2, 1, [1], None), (2, 2, [1, 0], []), (1, 2, [0, 0], [5])])
@pytest.mark.parametrize("H,D,T,S,L", [(2, 64, 16, 1, 6), (3, 128, 33, 0, 7), (1, 64, 1, 3, 4), (2, 128, 300, 2, 40)])
def test_fork_copies_the_chosen_frames(src_b, dst_b, parents, frames, H, D, T, S, L):
    import torch
    from paper_2603_17051_b200 import binding as A
    src, kx, vx, held = ring(A, src_b, H, D, T, S, L, 3, min(6, S + L) if L < 40 else 38, 70, poison=True)
    assert held >= 6
    for S2, L2 in ((0, max(1, held)), (2, 40)):
        dst = A.astro_kvcache_create(dst_b, H, D, T, S2, L2)
        A.astro_kvcache_append(dst, *(dev_bf16(synth.normal_bf16(3, (dst_b, 2 * T, H, D))) for _ in range(2)), 2) if L2 >= 2 else None
        p = None if parents is None else torch.tensor(parents, dtype=torch.int32, device="cuda")
        before = src.k_storage.clone()
        A.astro_kvcache_fork(dst, src, parents=p, frames=frames)
        assert torch.equal(src.k_storage, before)
        chosen = list(range(held)) if frames is None else frames
        sink, win, seen = A.astro_kvcache_query(dst)
        assert sink + win == len(chosen) and sink == min(S2, len(chosen))
        assert seen == A.astro_kvcache_query(src)[2]
        k, v = A.astro_kvcache_export(dst)
        rows = [parents[b] if parents else (0 if src_b == 1 else b) for b in range(dst_b)]
        tok = np.concatenate([np.arange(f * T, (f + 1) * T) for f in chosen]).astype(int) if chosen else np.zeros(0, int)
        for got, ref in ((k, kx), (v, vx)):
            assert np.array_equal(got.double().cpu().numpy(), ref[rows][:, tok])


def test_a_parent_outside_the_source_leaves_zeros():
    import torch
    from paper_2603_17051_b200 import binding as A
    src, kx, _, held = ring(A, 2, 2, 64, 20, 0, 4, 0, 3, 11)
    dst = A.astro_kvcache_create(4, 2, 64, 20, 0, 4)
    A.astro_kvcache_fork(dst, src, parents=torch.tensor([2, 1, -1, 2 ** 31 - 1], dtype=torch.int32, device="cuda"))
    k, v = A.astro_kvcache_export(dst)
    assert not k[0].any() and not v[2].any() and not k[3].any()
    assert np.array_equal(k[1].double().cpu().numpy(), kx[1])


def test_attention_of_the_forked_group_equals_that_of_the_shared_prefix():
    import torch
    from paper_2603_17051_b200 import binding as A
    src, _, _, held = ring(A, 1, 2, 128, 70, 1, 5, 2, 5, 21)
    G = 3
    dst = A.astro_kvcache_create(G, 2, 128, 70, 1, 5)
    A.astro_kvcache_fork(dst, src)
    q, k, v = (dev_bf16(synth.normal_bf16(600 + i, (G, 210, 2, 128))) for i in range(3))
    a, la = A.astro_chunk_attn_fwd(src, q, k, v, 0.1)
    b, lb = A.astro_chunk_attn_fwd(dst, q, k, v, 0.1)
    # the same keys in another order of the ring: two roundings of P and of the result each
    assert (a.float() - b.float()).abs().max() <= 1e-2 and (la - lb).abs().max() <= 1e-4
    A.astro_kvcache_evict(dst, 1)                        # the copies go on by themselves
    A.astro_kvcache_append(dst, k[:, :70].contiguous(), v[:, :70].contiguous(), 1)
    ke, _ = A.astro_kvcache_export(dst)
    assert torch.equal(ke[:, -70:], k[:, :70]) and A.astro_kvcache_query(src)[1] == 4


def test_refusals_leave_the_destination_alone():
    import torch
    from paper_2603_17051_b200 import binding as A
    src, _, _, held = ring(A, 2, 2, 64, 20, 0, 4, 0, 3, 31)
    make = lambda *a, **k: A.astro_kvcache_create(*a, **k)  # noqa: E731
    dst = make(2, 2, 64, 20, 0, 3)
    A.astro_kvcache_fork(dst, src)
    for other, kw, status in ((make(2, 1, 64, 20, 0, 3), {}, 2), (make(2, 2, 128, 20, 0, 3), {}, 2), (make(2, 2, 64, 21, 0, 3), {}, 2),
                              (make(3, 2, 64, 20, 0, 3), {}, 2), (make(2, 2, 64, 20, 0, 2), {}, 4), (dst, dict(frames=[3]), 2),
                              (dst, dict(frames=[-1]), 2), (src, {}, 2), (make(2, 2, 64, 20, 0, 4, k_storage=src.v_storage, v_storage=dst.k_storage.new_empty(src.k_storage.shape)), {}, 2)):
        with pytest.raises(A.AstroError) as e:
            A.astro_kvcache_fork(other, src, **kw)
        assert e.value.status == status
    assert A.astro_kvcache_query(dst)[:2] == (0, 3)
    for parents in (torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(ValueError):
            A.astro_kvcache_fork(dst, src, parents=parents)
