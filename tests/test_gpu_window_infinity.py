"""Window attention with one infinite element in a query or a key: every row and every gradient against the formula.  A query that sees a
score of +infinity (or NaN) is NaN; one that sees -infinity has the result without that key."""
import pytest

from attn_bounds import check, head

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("what", ["q", "k"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
@pytest.mark.parametrize("block,window,sink,at", [(1, 100, 2, 210), (100, 200, 50, 210), (1, 100, 2, 1), (100, 200, 50, 0), (1, 400, 0, 399), (1, 3, 0, 128)])
def test_one_infinite_element(D, what, value, block, window, sink, at):
    import torch
    from paper_2603_17051_b200 import binding as A
    n, H, scale, e = 400, 2, 0.125, 9
    g = torch.Generator(device="cuda").manual_seed(at + D)
    q, k, v, d_o = (torch.randn(1, n, H, D, generator=g, device="cuda").bfloat16() for _ in range(4))
    form = dict(block_tokens=block, window_tokens=window, sink_tokens=sink)
    clean = A.astro_window_attn_fwd(q, k, v, scale, **form)
    clean += A.astro_window_attn_bwd(q, k, v, *clean, d_o, scale, **form)
    (q if what == "q" else k)[0, at, 0, e] = value
    o, lse = A.astro_window_attn_fwd(q, k, v, scale, **form)
    dq, dk, dv = A.astro_window_attn_bwd(q, k, v, o, lse, d_o, scale, **form)
    A.astro_last_device_status()
    for got, was in zip((o, lse.transpose(1, 2), dq, dk, dv), (clean[0], clean[1].transpose(1, 2), *clean[2:])):
        assert torch.equal(got[:, :, 1], was[:, :, 1])                       # the other head

    qq, kk, vv, gg = (t[0, :, 0].double() for t in (q, k, v, d_o))
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    end = (i // block + 1) * block
    see = (j < end) & ((j < sink) | (j >= end - window))
    x = scale * (qq @ kk.T)
    lost = (see & (x.isnan() | (x == torch.inf))).any(1) | (see.sum(1) == (see & (x == -torch.inf)).sum(1))
    gone = see & (x == -torch.inf) & ~lost[:, None]                          # pairs without weight
    assert lost.any() or gone.any()                                          # one alone where a single query sees the key
    want = head(qq.nan_to_num(posinf=0.0, neginf=0.0), kk.nan_to_num(posinf=0.0, neginf=0.0), vv, scale, see & ~gone & ~lost[:, None], gg)
    nan = float("nan")

    def expect(name, rows, more=None):
        value_, bound = (t.clone() for t in want[name])
        value_[rows] = nan
        if more is not None:
            value_[more, e] = nan
        return value_, bound

    check(o[0, :, 0], expect("o", lost), "O")
    assert not lse[0, 0, lost].isfinite().any()
    check(lse[0, 0, ~lost], tuple(t[~lost] for t in want["lse"]), "LSE")
    check(dq[0, :, 0], expect("dq", lost, gone.any(1)), "dQ")                # a weight of 0 times an infinite key: NaN, by the formula
    keys = see[lost].any(0)                                                  # what a lost query has a part in
    check(dk[0, :, 0], expect("dk", keys), "dK")
    check(dv[0, :, 0], expect("dv", keys), "dV")
