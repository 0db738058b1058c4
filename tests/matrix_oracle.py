"""Plain forms of the orthogonalised update and of the 8-bit linear layer, in 64 bits."""
import numpy as np

COEFFS = (3.4445, -4.7750, 2.0315)
U16 = 2.0 ** -11  # a binary16 rounding is off by at most this, relative to the value
TINY16 = 2.0 ** -25  # ... or this, below the normal numbers


def f16(x):
    return np.asarray(x, np.float64).astype(np.float16).astype(np.float64)


def orthogonal(u, steps=5, copies=0):
    """The definition; with copies, the products' operands rounded as the library states (X itself is
    not): to binary16 in its scales, or, in all but the first `copies - 1` steps and throughout where
    the matrix has at most 64 rows or columns, to the sum of two such numbers."""
    a, b, c = COEFFS
    u = np.asarray(u, np.float64)
    size = np.sqrt((u * u).sum())
    if size == 0:
        return u
    x = (u.T if u.shape[0] > u.shape[1] else u) / size
    for i in range(steps):
        if not copies:
            r = lambda v, s: v
        elif i < copies - 1 and x.shape[0] > 64:
            r = lambda v, s: f16(v * s) / s
        else:
            r = lambda v, s: (f16(v * s) + f16(v * s - f16(v * s))) / s
        h = r(x, 2.0 ** 15)
        s = r(h @ h.T, 2.0 ** 15)
        x = a * x + r(b * s + c * (s @ s), 2.0 ** 14) @ h
    return x.T if u.shape[0] > u.shape[1] else x


def orthogonal_tolerance(u, steps=5, single=5):
    """How far (Frobenius norm) the library's FP32 result may be from the exact one, when its first
    `single` steps multiply single copies.

    Its error is that of the stated roundings of the operands, whose size the emulation
    gives.  Another summation order draws other roundings of the same size: the norms of
    two such draws over n independent elements differ by a few times n^-1/2 of themselves,
    and a matrix of a few elements can have one draw near zero, so three times the
    emulation's error, and one half step (2^-11) per product chain of the result for the
    draws that come out near zero.  Where the last step multiplies pairs, the emulation has 2^-22 of
    each operand; FP32 sums of 3 n / 16 instructions' products are up to 2^-24 of their
    magnitudes off at each, twice in B and once in X, and a step passes an error on at most 3.44 times
    as large: 2^-24 (3 n / 16) times 16 covers the steps of pairs, beside 2^-12 for those before them."""
    e = orthogonal(u, steps)
    off = np.linalg.norm(orthogonal(u, steps, copies=single + 1) - e)
    if single < steps or min(u.shape) <= 64:
        return 3 * off + (U16 / 2 + 3 * max(u.shape) * 2.0 ** -24) * np.linalg.norm(e)
    return 3 * off + 2 * U16 * np.linalg.norm(e)


def muon(w, v, g, lr, momentum, wd, scale, nesterov, steps=5):
    """(w, v, u): the new weights, unrounded, the new momentum, unrounded, and what is orthogonalised."""
    w, v, g = (np.asarray(t, np.float64) for t in (w, v, g))
    momentum = float(np.float32(momentum))
    new = momentum * v + g
    kept = f16(new)
    u = g + momentum * kept if nesterov else kept
    return w - lr * (scale * orthogonal(u, steps) + wd * w), new, u


def quantize(x):
    """(q, scale) of the rows of a binary16 matrix."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        a = np.abs(x).max(axis=1)
        q = np.rint(127 * x / a[:, None])  # a tie is exact in 64 bits, anything else 2^-19 away from one
        good = np.isfinite(a) & (a > 0)
        return np.where(good[:, None], q, 0).astype(np.int8), np.where(np.isfinite(a), a / 127, np.nan)


def linear(x, sx, w, sw, bias=None):
    """(y, slack): the exact result and what FP32 arithmetic may add to it before the rounding."""
    x, w, sx, sw = (np.asarray(t, np.float64) for t in (x, w, sx, sw))
    acc = x @ w.T  # exact: integers below 2^53
    s = sx[:, None] * sw[None, :]
    y = acc * s
    k = x.shape[1]
    # the scales' product and the sum's conversion: half a step of FP32 each, and the FMA one more
    slack = 3 * 2.0 ** -24 * np.abs(y)
    if k > 1024:  # partial sums past 2^24 may be rounded or cut, once per product of 16 terms
        slack = slack + (k / 16) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T) * s
    if bias is not None:
        y = y + np.asarray(bias, np.float64)[None, :]
        slack = slack + 2.0 ** -24 * np.abs(y)
    return y, slack
