"""Attention over lists of key blocks on inputs at the edge of the numbers: infinite scores, NaN and infinities in listed and in
unlisted blocks."""
import numpy as np
import pytest

from helpers import f64
from oracle import sparse_attn as orc
from test_gpu_sparse_attn import HALF, reference

pytestmark = pytest.mark.gpu
N_Q = [1, 2, 5, 40, 300]     # single queries, pairs, one tile (5 with long lists: split ones), several tiles


def inputs(D, n_q, n_kc, seed, H=2):
    import torch
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((1, n, H, D), generator=g).bfloat16() for n in (n_q, n_kc, n_kc)]


def forward(q, k, v, blocks, block, scale, mode=0):
    import torch
    from paper_2603_17051_b200 import binding as A
    A.astro_debug_forward_mode(mode)
    try:
        o, lse = A.astro_sparse_attn_fwd(None, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(blocks).cuda(), block, scale)
    finally:
        A.astro_debug_forward_mode(0)
    A.astro_last_device_status()
    return o, lse


def wanted(q, k, v, blocks, n_kc, block, scale, d_o=None):
    none = np.zeros((1, 0, q.shape[2], q.shape[3]))
    ranges = orc.key_blocks(0, 1, n_kc, block)
    with np.errstate(all="ignore"):
        return reference(*(x.double().numpy() for x in (q, k, v)), none, none, blocks, ranges, scale, 0, d_o)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", N_Q)
@pytest.mark.parametrize("low", [-100.0, -600.0])
def test_minus_infinity_in_every_score_of_the_first_tile(D, n_q, low):
    """A block masked by -infinity in one element of its keys comes first; the scores behind it are far below zero, where
    exp(score) without a reference of their own would be zero."""
    import torch
    block, n_kc, scale = 128, 384, 1.0
    q, k, v = inputs(D, n_q, n_kc, 7 + n_q)
    q[..., 0] = 1.0
    k[:, :128, :, 0] = -float("inf")
    k[:, 128:, :, 0] = low
    blocks = np.broadcast_to(np.array([0, 2, 1] + [-1] * 60, np.int32), (1, 2, -(-n_q // 128), 63)).copy()
    ref, o_abs = wanted(q, k, v, blocks, n_kc, block, scale)
    score = (D + 8) * 2.0 ** -24 * (abs(low) + 60.0)     # fp32 sums whose parts reach |low| + sum |q_d k_d|, the exponent's rounding
    for mode in (0, 1):
        o, lse = forward(q, k, v, blocks, block, scale, mode)
        assert torch.isfinite(lse).all()
        assert np.abs(f64(lse) - ref[1]).max() <= score + 2.0 ** -22 * (abs(low) + 60.0)
        err = np.abs(f64(o) - ref[0])
        assert (err <= HALF * np.abs(ref[0]) + (HALF + 2 * score) * o_abs * (1 + HALF)).all()
    # a list that names nothing but the masked block has no weight to share out
    only = np.where(blocks == 0, 0, -1).astype(np.int32)
    o, lse = forward(q, k, v, only, block, scale)
    assert torch.isneginf(lse).all() and not o.any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", N_Q)
@pytest.mark.parametrize("what", ["k nan", "k inf", "v nan", "v inf", "v both"])
def test_nan_and_infinities_reach_the_queries_that_name_their_block_and_no_other(D, n_q, what):
    import torch
    from paper_2603_17051_b200 import binding as A
    block, n_kc, scale = 32, 400, D ** -0.5
    q, k, v = inputs(D, n_q, n_kc, 70 + n_q)
    d_o = torch.randn(q.shape, generator=torch.Generator().manual_seed(1)).bfloat16()
    q[..., 3] = q[..., 3].abs() + 0.25                   # no zero beside the infinity: 0 * inf would be one more NaN
    bad, value = (k if what[0] == "k" else v), float("nan") if "nan" in what else float("inf")
    bad[0, 5 * 32 + 7, 0, 3] = value                     # head 0, block 5; head 1 stays clean
    if what == "v both":
        bad[0, 5 * 32 + 9, 0, 3] = -value
    nqb = -(-n_q // 128)
    blocks = np.zeros((1, 2, nqb, 6), np.int32)
    for i in range(nqb):
        blocks[0, :, i] = [0, 5, 2, 9, 12, 1] if i % 2 == 0 else [3, 4, 12, -1, 6, 0]
    clean = np.where(blocks == 5, 7, blocks).astype(np.int32)
    for lists_ in (blocks, clean):
        ref, _ = wanted(q, k, v, lists_, n_kc, block, scale, d_o.double().numpy())
        o, lse = forward(q, k, v, lists_, block, scale)
        grads = A.astro_sparse_attn_bwd(None, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(lists_).cuda(), block, o, lse, d_o.cuda(), scale)
        A.astro_last_device_status()
        for got, want, tag in zip((o, lse) + grads, ref, ("O", "LSE", "dQ", "dK", "dV")):
            got = f64(got)
            whole = np.isfinite(want)
            if lists_ is clean:
                assert whole.all()
            # what is finite in the definition stays so; what is not does not turn into a number.  (Which of NaN and the infinities
            # a sum ends in is the definition's for O and LSE alone: gradients pass through delta = dO . O.)
            assert np.array_equal(np.isfinite(got), whole), tag
            if tag in ("O", "LSE"):
                assert np.array_equal(np.isnan(got), np.isnan(want)), tag
                assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), tag
            err = np.linalg.norm(got[whole] - want[whole])
            assert err <= 1e-2 * np.linalg.norm(want[whole]) + 1e-6 * np.sqrt(whole.sum()), (tag, err)
