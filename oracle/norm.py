"""The norms, gate and scaled residual between two blocks, in fp64.

Oracle - test infrastructure only (see the package docstring).

    fh = (f - mean f) / sqrt(var f + eps)   (layer), f / sqrt(mean f^2 + eps)   (rms)
    u = fh w_post + b_post,  y = res_scale x + g u,  z = yh w_pre + b_pre

With <v> a row's mean, t = dy + r_y (dz w_pre - <dz w_pre> - yh <dz w_pre yh>) is the gradient of y (the <dz w_pre>
term for layer only), dx = res_scale t, dg = u t, du = g t, and df follows from du as t does from dz.

``block`` gives beside each result a bound: how far a computation in fp32 may be off that adds a row's D values in any
order and rounds results once (half: the half step of x's type).
"""

from __future__ import annotations

import numpy as np


def _unit(v, layer, eps):
    mean = v.mean(axis=1, keepdims=True) if layer else np.zeros((v.shape[0], 1))
    r = 1.0 / np.sqrt(((v - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    return (v - mean) * r, r


def _unit_grad(d, hat, r, layer):
    m = d.mean(axis=1, keepdims=True) if layer else 0.0
    return r * (d - m - hat * (d * hat).mean(axis=1, keepdims=True))


def block(x, f, *, w_post=None, b_post=None, w_pre=None, b_pre=None, gate=None, sigmoid=False, res_scale=1.0,
          layer=True, eps=1e-5, dy=None, dz=None, half=2.0 ** -24):
    """(results, bounds): dicts of y, z and, with dy and dz, dx, df, dgate, dw_post, db_post, dw_pre, db_pre."""
    f64 = lambda v: None if v is None else np.asarray(v, dtype=np.float64)  # noqa: E731
    x, f, gate, dy, dz = (f64(v) for v in (x, f, gate, dy, dz))
    n, D = x.shape
    one, zero = np.ones(D), np.zeros(D)
    w1, b1, w2, b2 = (f64(v) if v is not None else e for v, e in zip((w_post, b_post, w_pre, b_pre),
                                                                     (one, zero, one, zero)))
    g = np.ones((1, D)) if gate is None else 1.0 / (1.0 + np.exp(-gate)) if sigmoid else np.atleast_2d(gate)
    g = np.broadcast_to(g, x.shape)
    fh, rf = _unit(f, layer, eps)
    u = fh * w1 + b1
    y = res_scale * x + g * u
    yh, ry = _unit(y, layer, eps)
    z = yh * w2 + b2
    top = lambda v: np.abs(v).max(axis=1, keepdims=True, initial=0.0)  # noqa: E731
    e = (D + 32) * 2.0 ** -24  # a row's sum, and the handful of roundings around it
    # a normalised value is off by e times the row's size before the mean went, in units of its spread
    e_fh = 4 * e * (1 + top(f) * rf) * (1 + np.abs(fh))
    e_u = np.abs(w1) * e_fh + e * (np.abs(u) + np.abs(b1))
    e_y = np.abs(g) * e_u + e * (np.abs(res_scale * x) + np.abs(g * u))
    e_yh = (ry * (e_y + top(e_y)) + 4 * e * (1 + top(y) * ry)) * (1 + np.abs(yh)) * (1 + np.abs(yh))
    r = {"y": y, "z": z}
    b = {"y": e_y + half * np.abs(y), "z": np.abs(w2) * e_yh + e * np.abs(b2) + half * np.abs(z)}
    if dz is None:
        return r, b
    d2 = dz * w2
    t = dy + _unit_grad(d2, yh, ry, layer)
    # the gradient through a norm: its terms' roundings, and what yh (and r_y, as much) is off
    e_t = e * np.abs(dy) + ry * (8 * e * (np.abs(d2) + top(d2) * (1 + np.abs(yh)) * (1 + top(yh)))
                                 + 2 * top(d2) * (top(e_yh) * (1 + np.abs(yh)) + e_yh * (1 + top(yh)))
                                 + top(e_yh) * (np.abs(d2) + top(d2) * (1 + np.abs(yh))))
    du, dg = g * t, u * t
    d1 = du * w1
    df = _unit_grad(d1, fh, rf, layer)
    e_du = np.abs(g) * e_t + e * np.abs(du)
    e_d1 = np.abs(w1) * e_du + e * np.abs(d1)
    e_df = rf * (e_d1 + top(e_d1) * (1 + np.abs(fh)) * (1 + top(fh))
                 + 8 * e * (np.abs(d1) + top(d1) * (1 + np.abs(fh)) * (1 + top(fh)))
                 + 2 * top(d1) * (top(e_fh) * (1 + np.abs(fh)) + e_fh * (1 + top(fh)))
                 + top(e_fh) * (np.abs(d1) + top(d1) * (1 + np.abs(fh))))
    e_dg = np.abs(u) * e_t + np.abs(t) * e_u + e * np.abs(dg)
    r.update(dx=res_scale * t, df=df)
    b.update(dx=abs(res_scale) * e_t + half * np.abs(r["dx"]), df=e_df + half * np.abs(df))
    if gate is not None:
        if gate.ndim == 1:
            r["dgate"], b["dgate"] = dg.sum(axis=0), sums(e_dg, dg)
        else:
            k = g * (1 - g) if sigmoid else np.ones_like(g)
            r["dgate"] = dg * k
            # 1 - g loses what g carries next to 1
            b["dgate"] = e_dg * k + 2.0 ** -22 * np.abs(dg) + half * np.abs(r["dgate"])
    for name, v, ev, given in (("dw_post", du * fh, e_du * np.abs(fh) + np.abs(du) * e_fh, w_post),
                               ("db_post", du, e_du, b_post),
                               ("dw_pre", dz * yh, np.abs(dz) * e_yh, w_pre), ("db_pre", dz, 0 * dz, b_pre)):
        if given is not None:
            r[name], b[name] = v.sum(axis=0), sums(ev, v)
    return r, b



def sums(err, v):
    """The bound of a column's fp32 sum: its terms', and the additions' (chains of at most 4,096)."""
    return err.sum(axis=0) + (min(v.shape[0], 4096) + 4) * 2.0 ** -24 * np.abs(v).sum(axis=0)


# What fp32 adds to a whole row (or a parameter's gradient), in its size.  A result is six stages from the inputs (f's
# norm, y, y's norm, t, du and df, or a product with one of them), each at most eight roundings and a row's mean of at
# most 32 dependent additions: 40 half steps of its operands' size.  A norm's Jacobian is a projection over the spread,
# so what a stage takes over is not enlarged but by the weights, gates and scales, which stay within a factor of four
# for parameters around one: 6 * 40 * 4 * 2^-24 < 2^-14.
ROW = 2.0 ** -14


def normwise(got, ref, half):
    """Each result's largest error over its tolerance: a row of y, z, dx, df (and of a gradient of the gate's rows)
    against ROW and its rounding, a parameter's gradient as a whole against ROW times the root of the rows' number (a
    sum of n terms of random sign is that much smaller than its terms).  Above 1 is outside."""
    n = len(ref["y"])
    out = {}
    for name, r in ref.items():
        x = np.asarray(got[name], dtype=np.float64)
        tol = half + ROW if r.ndim == 2 else ROW * np.sqrt(n)
        out[name] = float((np.linalg.norm(x - r, axis=-1) / (tol * np.linalg.norm(r, axis=-1))).max())
    return out
