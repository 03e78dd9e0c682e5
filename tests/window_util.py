"""64-bit reference of attention with a sliding window and first tokens that stay visible,
with bounds on how far the kernels may be from it: those of tests/train_ops_util.py, over
the keys that a query sees."""
import math

import numpy as np

from train_ops_util import H, U


def window_reference(q, k, v, lens, window, sinks, scale, dout=None, only=None):
    """(dict of fp64 arrays out, lse, dq, dk, dv, dict of their bounds for no bf16 rounding and for
    bf16 rounding); row by row, over visible keys only.  only: the sequences to look at (the
    others' rows stay 0)."""
    q, k, v = (np.asarray(x.detach().double().cpu()) for x in (q, k, v))
    t, hq, d = q.shape
    g = hq // k.shape[1]
    res = {"out": np.zeros_like(q), "lse": np.zeros((hq, t))}
    tol = {"out": np.zeros((2,) + q.shape), "lse": np.zeros((2, hq, t))}
    if dout is not None:
        do = np.asarray(dout.detach().double().cpu())
        for n, x in (("dq", q), ("dk", k), ("dv", v)):
            res[n], tol[n] = np.zeros_like(x), np.zeros((2,) + x.shape)
    rounds = np.array([0.0, H])

    def finite(x):
        return np.abs(np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0))
    with np.errstate(invalid="ignore", over="ignore"):
        start = 0
        for s, n in enumerate(lens):
            for i in range(n) if only is None or s in only else ():
                lo = max(0, i - window + 1)
                seen = start + np.concatenate([np.arange(min(sinks, lo)), np.arange(lo, i + 1)])
                at, m = start + i, len(seen)
                for h in range(hq):
                    kh = h // g
                    ks, vs = k[seen, kh], v[seen, kh]
                    x = scale * (ks @ q[at, h])
                    top = x.max()
                    e = np.exp(x - top)
                    p = e / e.sum()
                    res["out"][at, h] = o = p @ vs
                    res["lse"][h, at] = top + math.log(e.sum()) if np.isfinite(top) else top
                    ak, av_, aq = finite(ks), finite(vs), finite(q[at, h])
                    eps = 2 * (d + 8) * U * abs(scale) * (ak @ aq).max() + (m + 64) * U
                    av = p @ av_
                    for r, hr in enumerate(rounds):
                        tol["out"][r, at, h] = (eps + hr) * av + hr * np.abs(o)
                        tol["lse"][r, h, at] = eps + 4 * U * abs(res["lse"][h, at])
                    if dout is None:
                        continue
                    dd = do[at, h]
                    ds = p * (vs @ dd - dd @ o)
                    res["dq"][at, h] = scale * (ds @ ks)
                    res["dk"][seen, kh] += scale * np.outer(ds, q[at, h])
                    res["dv"][seen, kh] += np.outer(p, dd)
                    mag = p * (av_ @ np.abs(dd) + np.abs(dd) @ av)
                    for r, hr in enumerate(rounds):
                        off = hr * np.abs(ds) + hr * p * (np.abs(dd) @ np.abs(o)) + 2 * eps * mag
                        tol["dq"][r, at, h] = abs(scale) * (off @ ak) + hr * np.abs(res["dq"][at, h])
                        tol["dk"][r, seen, kh] += abs(scale) * np.outer(off, aq)
                        tol["dv"][r, seen, kh] += (eps + hr) * np.outer(p, np.abs(dd))
            start += n
    if dout is not None:
        for n in ("dk", "dv"):
            for r, hr in enumerate(rounds):
                tol[n][r] += hr * np.abs(res[n]) + g * max(lens, default=0) * U * np.abs(res[n])
    return res, tol
