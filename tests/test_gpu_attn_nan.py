"""NaN in an operand of the dense attention reaches every gradient that it belongs to."""
import numpy as np
import pytest

from helpers import f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("row", [0, 1, 2, 3, 4, 7, 16, 40, 131])
def test_a_nan_in_one_query_shows_in_the_gradient_of_every_key(D, row):
    """P of that query is NaN for every key, so dK and dV are NaN throughout its head (in whichever column of a tile it stands) and
    dQ in its own row alone."""
    import torch
    from paper_2603_17051_b200 import binding as A
    g = torch.Generator().manual_seed(row)
    q, k, v, d_o = (torch.randn((1, n, 2, D), generator=g).bfloat16().cuda() for n in (140, 90, 90, 140))
    q[0, row, 0, 5] = float("nan")
    o, lse = A.astro_chunk_attn_fwd(None, q, k, v, D ** -0.5)
    dq, dk, dv = (f64(x) for x in A.astro_chunk_attn_bwd(None, q, k, v, o, lse, d_o, D ** -0.5))
    A.astro_last_device_status()
    assert np.isnan(dk[:, :, 0]).all() and np.isnan(dv[:, :, 0]).all() and np.isfinite(dk[:, :, 1]).all() and np.isfinite(dv[:, :, 1]).all()
    bad = np.isnan(dq).all(-1)
    assert bad[0, row, 0] and bad.sum() == 1 and np.isfinite(np.delete(dq, row, 1)).all()
