"""64-bit reference of the norm and rotation of query and key heads, with a bound on how far
the kernels may be from it, element by element.  u = 2^-24 is the rounding of fp32, h = 2^-8
that of bf16 results (u of fp32 ones):

* 1 / sqrt(mean + eps) is made in 64 bits and rounded to fp32 (u, and 2^-40 for its
  Newton step); x times it times w: two roundings;
* cos and sin: the angle, below pi / 4, is rounded twice (u each), polynomials of it are
  rounded a few times at the size of 1: within 5 u together; and the angle itself, made in 64
  bits in three roundings, is off by |t| 2^-51;
* a turned feature: two products and a sum (u each of the products' sizes);
* a mean or a sum of n terms adds n u of the sum of their sizes at most.

The angles are made in numpy's long double (64 bits of mantissa)."""
import numpy as np

U = 2.0 ** -24
H = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def members(dim, pairs, adjacent):
    """Features of each turning pair."""
    i = np.arange(pairs)
    return (2 * i, 2 * i + 1) if adjacent else (i, i + pairs)


def angles(positions, freqs, axes):
    """[tokens, pairs] in long double; positions [axes, tokens]."""
    f = np.asarray(freqs, dtype=np.float64).astype(np.longdouble)
    a = np.zeros(len(freqs), int) if axes is None else np.asarray(axes)
    return positions.astype(np.longdouble)[a].T * f[None, :]


def _turn(x, ex, t, pairs, adjacent, back):
    """(turned x, bound) of x with bound ex, [tokens, heads, dim]."""
    y, ey = x.copy(), ex.copy()
    if pairs == 0:
        return y, ey
    c, s = np.cos(t).astype(np.float64)[:, None], np.sin(t).astype(np.float64)[:, None]
    if back:
        s = -s
    a, b = members(x.shape[2], pairs, adjacent)
    off = (5 * U + np.abs(t).astype(np.float64)[:, None] * 2.0 ** -51 + 2 * U) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    ey[..., a] = ex[..., a] * np.abs(c) + ex[..., b] * np.abs(s) + off
    ey[..., b] = ex[..., a] * np.abs(s) + ex[..., b] * np.abs(c) + off
    return y, ey


def reference(x, w, positions, freqs, axes, adjacent, norm, eps, kind, g=None):
    """{"y", "dx", "dw"}: (value, bound) of one operand x [tokens, heads, dim], fp64."""
    pairs, dim, h = len(freqs), x.shape[2], H[kind]
    t = angles(positions, freqs, axes) if pairs else None
    ww = np.ones(dim) if w is None else w
    with np.errstate(all="ignore"):
        if norm:
            r = 1.0 / np.sqrt((x * x).mean(2, keepdims=True) + eps)
            n = x * r * ww
        else:
            r, n = np.ones(x.shape[:2] + (1,)), x
        y, ey = _turn(n, 4 * U * np.abs(n), t, pairs, adjacent, False)
        res = {"y": (y, ey + h * np.abs(y))}
        if g is None:
            return res
        z, ez = _turn(g, np.zeros_like(g), t, pairs, adjacent, True)
        if not norm:
            return res | {"dx": (z, ez + h * np.abs(z))}
        xh = x * r
        dw = (z * xh).sum((0, 1))
        rows = x.shape[0] * x.shape[1]
        edw = (ez * np.abs(xh)).sum((0, 1)) + (4 * U + (rows + 16) * U) * (np.abs(z * xh)).sum((0, 1))
        v, ev = z * ww, ez * np.abs(ww) + U * np.abs(z * ww)
        m = (v * xh).mean(2, keepdims=True)
        em = (ev * np.abs(xh)).mean(2, keepdims=True) + (4 * U + (dim + 8) * U) * np.abs(v * xh).mean(2, keepdims=True)
        dx = r * (v - xh * m)
        edx = r * (ev + np.abs(xh) * em + 8 * U * (np.abs(v) + np.abs(xh * m)))
    return res | {"dx": (dx, edx + h * np.abs(dx)), "dw": (dw, edw + U * np.abs(dw))}


def assert_close(name, got, want_and_bound):
    want, tol = want_and_bound
    got = np.asarray(got.detach().double().cpu())
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine), f"{name}: other places are finite"
    off = np.abs(got[fine] - want[fine]) - tol[fine]
    worst = off.max() if off.size else 0.0
    assert worst <= 1e-37, f"{name}: {worst:.3e} outside its bound"
