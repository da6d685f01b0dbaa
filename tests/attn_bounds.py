"""Attention of one head in 64 bits, forward and backward, with a bound on the error of each result for kernels that multiply
in bf16 and sum in fp32.

Half a step of bf16 is H = 2^-8 of a value.  The weights are rounded to it before they meet V (forward) or dO (dV), dS before it
meets K or Q, every output once more; delta = dO . O is taken from the rounded O.  What fp32 adds (sums, exp2 to a few 1e-7, a
polynomial exp2 to 7.6e-5 in dK/dV) stays below H / 32, which the bounds allow beside H.
"""
import torch

H = 2.0 ** -8
SLACK = 1.0 + 1.0 / 32


def head(q, k, v, scale, see=None, d_o=None, v_size=None):
    """q [n, D], k, v [m, D] in fp64; see [n, m] or None; returns {name: (value, bound)}.  LSE's bound is absolute 2e-6 per unit
    of the largest score and of itself (fp32 sums and products)."""
    x = scale * (q @ k.T)
    size = scale * (q.abs() @ k.abs().T)                     # what the fp32 sum of a score can be off by is relative to this
    if see is not None:
        x = x.masked_fill(~see, -torch.inf)
        size = size.masked_fill(~see, 0.0)
    lse = torch.logsumexp(x, 1)
    p = torch.where(x == -torch.inf, 0.0, torch.exp(x - lse[:, None]))
    p = torch.nan_to_num(p, nan=0.0) if see is not None else p
    fp32 = 2.0 ** -20 * size.amax(1, keepdim=True)           # relative error of a weight from its score
    o = p @ v
    o_bound = SLACK * ((H + fp32) * (p @ v.abs()) + H * o.abs()) + 1e-7
    out = {"o": (o, o_bound), "lse": (lse, 1e-6 + fp32[:, 0] + 2.0 ** -22 * lse.abs())}
    if d_o is not None:
        dp = d_o @ v.T
        delta = (d_o * o).sum(1, keepdim=True)
        delta_err = (d_o.abs() * o_bound).sum(1, keepdim=True)
        dp_size = d_o.abs() @ v.abs().T
        ds = p * (dp - delta)
        ds_err = (H + fp32) * ds.abs() + p * (delta_err + 2.0 ** -20 * dp_size)
        dq, dk, dv = scale * (ds @ k), scale * (ds.T @ q), p.T @ d_o
        out["dq"] = (dq, SLACK * (scale * (ds_err @ k.abs()) + H * dq.abs()) + 1e-7)
        out["dk"] = (dk, SLACK * (scale * (ds_err.T @ q.abs()) + H * dk.abs()) + 1e-7)
        out["dv"] = (dv, SLACK * (((H + fp32) * p).T @ d_o.abs() + H * dv.abs()) + 1e-7)
    return out


def check(got, want, tag=""):
    """`got` against (value, bound): equal where the value is infinite, NaN where it is NaN."""
    value, bound = want
    got = got.double()
    assert got.shape == value.shape, tag
    finite = value.isfinite()
    same = (got == value) | (got.isnan() & value.isnan())
    assert bool((finite | same).all()), "%s: infinities and NaN differ" % tag
    over = ((got - value).abs() - bound)[finite]
    if over.numel():
        assert not bool(over.isnan().any()) and over.max().item() <= 0, "%s: %.3e beyond its bound" % (tag, over.max().item())
