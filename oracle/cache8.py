"""fp64 oracle of rows held in 8 bits: a power of two per row and e4m3 values."""
import numpy as np

LOWEST_EXP = -124


def e4m3(y):
    """Rounded to the nearest e4m3 number (|y| <= 448), ties to even: 3 bits behind the leading one, multiples of 2^-9 below
    2^-6.  NaN stays NaN."""
    a = np.abs(y)
    _, k = np.frexp(np.where(np.isfinite(a), a, 0.0))          # a = f 2^k, f in [0.5, 1)
    step = np.exp2(np.maximum(k - 1, -6) - 3.0)
    return np.rint(y / step) * step


def exponents(x):
    """e of every row [..., D]: smallest with max |x| <= 448 * 2^e over the finite elements."""
    x = np.asarray(x, dtype=np.float64)
    top = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    f, k = np.frexp(top)
    e = np.where(f <= 0.875, k - 9, k - 8)                     # 448 = 0.875 * 2^9
    return np.maximum(np.where(top > 0, e, LOWEST_EXP), LOWEST_EXP)


def stands_for(x):
    """What the rows of x are after they have been written and read back (without a rounding of the reading)."""
    x = np.asarray(x, dtype=np.float64)
    e = exponents(x)[..., None]
    size = np.exp2(e.astype(np.float64))
    most = np.where(e == 120, 240.0, 448.0)                    # 256 * 2^120 is beyond every finite float
    with np.errstate(invalid="ignore"):
        return np.clip(e4m3(np.where(np.isfinite(x), x, np.nan) / size), -most, most) * size
