"""64-bit references of the training-step operators, with bounds on how far
the kernels may be from them.

The bounds follow from the number formats, element by element.  u = 2^-24 is
the rounding of fp32 and h = 2^-8 that of bf16 (0 for fp32 operands):

* a score is a sum of D products, so its exponent is off by at most
  g = 2 (D + 8) u max(c sum_d |q k|) (the factor 2: the log-sum-exp carries the
  same error), and a sum of n terms adds n u;
* the weights p and ds that enter a second matrix product are rounded once (h),
  the result once more;
* delta = do . o carries the rounding of o (h sum_d |do o|).
"""
import math

import numpy as np
import torch

U = 2.0 ** -24
H = 2.0 ** -8


def attention_reference(q, k, v, lens, causal, scale, dout=None):
    """dict of fp64 arrays out, lse, dq, dk, dv and, under "tol_*", the bound of
    each for bf16 rounding h = H and for none; row by row, over visible keys
    only, so nothing a row does not see can reach it."""
    q, k, v = (np.asarray(x.detach().double().cpu()) for x in (q, k, v))
    t, hq, d = q.shape
    hk = k.shape[1]
    g = hq // hk
    res = {"out": np.zeros_like(q), "lse": np.zeros((hq, t))}
    tol = {"out": np.zeros((2,) + q.shape), "lse": np.zeros((2, hq, t))}
    if dout is not None:
        do = np.asarray(dout.detach().double().cpu())
        for n, x in (("dq", q), ("dk", k), ("dv", v)):
            res[n] = np.zeros_like(x)
            tol[n] = np.zeros((2,) + x.shape)
    rounds = np.array([0.0, H])
    with np.errstate(invalid="ignore", over="ignore"):
        start = 0
        for n in lens:
            for h in range(hq):
                for i in range(n):
                    end = i + 1 if causal else n
                    at, seen = start + i, slice(start, start + end)
                    ks, vs, kh = k[seen, h // g], v[seen, h // g], h // g
                    s = scale * (ks @ q[at, h])
                    m = s.max()
                    e = np.exp(s - m)
                    p = e / e.sum()
                    res["out"][at, h] = p @ vs
                    res["lse"][h, at] = m + math.log(e.sum()) if np.isfinite(m) else m
                    # The bounds of finite results come from the finite operands.
                    ak, av_, aq = (np.abs(np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0))
                                   for x in (ks, vs, q[at, h]))
                    eps = 2 * (d + 8) * U * abs(scale) * (ak @ aq).max() + (n + 64) * U
                    av = p @ av_
                    for r, hr in enumerate(rounds):
                        tol["out"][r, at, h] = (eps + hr) * av + hr * np.abs(res["out"][at, h])
                        tol["lse"][r, h, at] = eps + 4 * U * abs(res["lse"][h, at])
                    if dout is None:
                        continue
                    dd = do[at, h]
                    dp = vs @ dd
                    delta = dd @ res["out"][at, h]
                    ds = p * (dp - delta)
                    res["dq"][at, h] = scale * (ds @ ks)
                    res["dk"][seen, kh] += scale * np.outer(ds, q[at, h])
                    res["dv"][seen, kh] += np.outer(p, dd)
                    # What ds may be off by: its own rounding, delta's, and fp32.
                    mag = p * (av_ @ np.abs(dd) + np.abs(dd) @ av)
                    for r, hr in enumerate(rounds):
                        off = hr * np.abs(ds) + hr * p * (np.abs(dd) @ np.abs(res["out"][at, h])) + 2 * eps * mag
                        tol["dq"][r, at, h] = abs(scale) * (off @ ak) + hr * np.abs(res["dq"][at, h])
                        tol["dk"][r, seen, kh] += abs(scale) * np.outer(off, aq)
                        tol["dv"][r, seen, kh] += (eps + hr) * np.outer(p, np.abs(dd))
            start += n
    if dout is not None:
        for n in ("dk", "dv"):
            for r, hr in enumerate(rounds):
                tol[n][r] += hr * np.abs(res[n]) + g * max(lens, default=0) * U * np.abs(res[n])
    return res, tol


def assert_within(name, got, want, tol):
    """|got - want| <= tol where want is finite; the same kind of value elsewhere.
    1e-30: results that underflow."""
    got = np.asarray(got.detach().double().cpu())
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine), f"{name}: other places are finite"
    off = np.abs(got[fine] - want[fine]) - np.asarray(tol)[fine]
    worst = off.max() if off.size else 0.0
    assert worst <= 1e-30, f"{name}: {worst:.3e} outside its bound"


def encode_reference(x):
    """(codes, exps) of the 8-bit checkpoint, group by group from the definition."""
    x = np.asarray(x.detach().double().cpu())
    rows, cols = x.shape
    pitch = -(-cols // 64) * 64
    codes = np.zeros((rows, pitch), np.int8)
    exps = np.zeros((rows, pitch // 64), np.int8)
    for i in range(rows):
        for g in range(pitch // 64):
            y = x[i, 64 * g:64 * g + 64]
            top = np.abs(y).max()
            if not np.isfinite(top):
                exps[i, g] = -128
                continue
            e = -126
            while e < 121 and np.rint(top * 2.0 ** -e) > 127:
                e += 1
            exps[i, g] = e
            codes[i, 64 * g:64 * g + len(y)] = np.clip(np.rint(y * 2.0 ** -e), -127, 127)
    return codes, exps


def decode_reference(codes, exps, cols):
    codes, exps = (np.asarray(x.cpu() if hasattr(x, "cpu") else x) for x in (codes, exps))
    step = np.where(exps == -128, np.nan, 2.0 ** exps.astype(np.float64))
    return (codes.astype(np.float64) * np.repeat(step, 64, axis=1))[:, :cols]


def logistic(x):
    return 1.0 / (1.0 + np.exp(-x))


GA, GB = 2.0 * math.sqrt(2.0 / math.pi), 0.044715


def act_reference(act, u, up=None):
    if act == "gelu":
        return u * logistic(GA * (u + GB * u ** 3))
    return u * logistic(u) * up


def act_grad_reference(act, dh, u, up=None):
    if act == "gelu":
        s = logistic(GA * (u + GB * u ** 3))
        return dh * (s + u * s * (1 - s) * GA * (1 + 3 * GB * u * u)), None
    s = logistic(u)
    return dh * up * s * (1 + u * (1 - s)), dh * u * s
