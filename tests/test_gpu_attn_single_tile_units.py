"""Dense forward over units of a single key tile, many per CTA: what one unit leaves in shared memory for the epilogue warps must
not be overwritten by the unit after the next."""
import numpy as np
import pytest

from helpers import dev_bf16, f64
from oracle.rolling_attn import bf16_bits_to_f64
from paper_2603_17051_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_kc", [128, 33])
def test_units_of_one_tile_keep_their_row_sums(D, n_kc):
    """8 x 40 x 3 units, seven or so per SM, the third query tile nearly empty.  Row sums differ from unit to unit by orders of
    magnitude (queries scaled by 0, 1/2 or 3), so a sum taken from another unit shows in O."""
    import torch
    from paper_2603_17051_b200 import binding as A
    B, H, n_q = 8, 40, 128 * 2 + 5
    q, k, v = (bf16_bits_to_f64(synth.normal_bf16(160 + i, (B, n, H, D))) for i, n in enumerate((n_q, n_kc, n_kc)))
    q *= np.array([0.0, 0.5, 3.0])[np.arange(B * n_q * H).reshape(B, n_q, H, 1) // 128 % 3]
    q, k, v = (torch.from_numpy(x).bfloat16() for x in (q, k, v))
    qf, kf, vf = (x.double() for x in (q, k, v))
    scale = D ** -0.5
    s = torch.einsum("bihd,bjhd->bhij", qf, kf) * scale
    p = torch.softmax(s, -1)
    want, lse_want = torch.einsum("bhij,bjhd->bihd", p, vf).numpy(), torch.logsumexp(s, -1).numpy()
    o_abs = torch.einsum("bhij,bjhd->bihd", p, vf.abs()).numpy()
    # fp32 scores: D products, partial sums below scale * sum |q_d k_d|; P and O rounded to bf16, half a step each
    score = (D + 8) * 2.0 ** -24 * 3 * 40.0 * max(1.0, scale * np.sqrt(D))
    half = 2.0 ** -8
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    first = None
    for _ in range(5):
        o, lse = A.astro_chunk_attn_fwd(None, q, k, v, scale)
        A.astro_last_device_status()
        if first is None:
            first = o.clone(), lse.clone()
            err = np.abs(f64(o) - want)
            assert (err <= half * np.abs(want) + (half + 2 * score) * o_abs * (1 + half)).all()
            assert np.abs(f64(lse) - lse_want).max() <= score + 2.0 ** -22 * np.abs(lse_want).max() + 1e-6
        assert torch.equal(o, first[0]) and torch.equal(lse, first[1])
