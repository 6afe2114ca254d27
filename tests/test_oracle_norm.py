"""CPU pins of the norms' normwise tolerance: an fp32 run of the formulas is inside it, and a backward that leaves out
one of its terms is not."""

import numpy as np
import pytest

from oracle import norm as ON
from synth.tensors import bf16_round, normal_tensor

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def backward(p, x, f, dy, dz, gate, sigmoid, layer, drop=(), a=0.75, eps=1e-5):
    """The formulas in fp32; drop: terms left out ('mean': <d>, 'hat': yh <d yh>, 'post mean' and 'post hat' the same of
    the norm after the block, 'gate': of du, 'norm': dz's way to y)."""
    one = np.float32(1)
    mean = lambda v: v.mean(axis=1, keepdims=True, dtype=np.float32)  # noqa: E731

    def unit(v):
        v = v - mean(v) if layer else v
        r = one / np.sqrt(mean(v * v) + np.float32(eps))
        return v * r, r

    def through(d, hat, r, which):
        m = mean(d) if layer and which + "mean" not in drop else np.float32(0)
        h = hat * mean(d * hat) if which + "hat" not in drop else np.float32(0)
        return r * (d - m - h)

    fh, rf = unit(f)
    u = fh * p["w_post"] + p["b_post"]
    g = one if gate is None else one / (one + np.exp(-gate)) if sigmoid else gate
    y = np.float32(a) * x + g * u
    yh, ry = unit(y)
    z = yh * p["w_pre"] + p["b_pre"]
    t = dy + (through(dz * p["w_pre"], yh, ry, "") if "norm" not in drop else np.float32(0))
    du, dg = t if "gate" in drop else g * t, u * t
    out = dict(y=y, z=z, dx=np.float32(a) * t, df=through(du * p["w_post"], fh, rf, "post "),
               dw_post=(du * fh).sum(0), db_post=du.sum(0), dw_pre=(dz * yh).sum(0), db_pre=dz.sum(0))
    if gate is not None:
        out["dgate"] = dg.sum(0) if gate.ndim == 1 else dg * g * (one - g) if sigmoid else dg
    return out


def case(D, dtype, gate, n=33):
    x, f, dy, dz = (normal_tensor((n, D), (D, t), dtype).astype(np.float32) for t in range(4))
    rng = np.random.default_rng(D)
    p = {k: (m + 0.3 * rng.normal(size=D)).astype(np.float32)
         for k, m in (("w_post", 1.0), ("b_post", 0.0), ("w_pre", 1.0), ("b_pre", 0.0))}
    g = None
    if gate == "vector":
        g = rng.normal(size=D).astype(np.float32)
    elif gate != "none":
        g = normal_tensor((n, D), (D, 9), dtype).astype(np.float32)
    return x, f, dy, dz, p, g


def worst(D, dtype, kind, gate, drop=()):
    x, f, dy, dz, p, g = case(D, dtype, gate)
    layer, sigmoid = kind == "layer", gate == "sigmoid"
    ref, _ = ON.block(x, f, gate=g, sigmoid=sigmoid, res_scale=0.75, layer=layer, eps=float(np.float32(1e-5)), dy=dy,
                      dz=dz, **p)
    got = backward(p, x, f, dy, dz, g, sigmoid, layer, drop)
    if dtype == "bf16":
        got = {k: bf16_round(v) if v.ndim == 2 else v for k, v in got.items()}
    return ON.normwise(got, ref, HALF[dtype])


@pytest.mark.parametrize("D", [64, 512, 8192])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("gate", ["none", "vector", "rows", "sigmoid"])
def test_a_backward_without_one_of_its_terms_is_outside(D, dtype, kind, gate):
    inside = worst(D, dtype, kind, gate)
    assert len(inside) == (8 if gate == "none" else 9) and max(inside.values()) < 1, inside
    hit = [("hat", ("dx", "df")), ("norm", ("dx", "df", "dw_post", "db_post")), ("post hat", ("df",))]
    if kind == "layer":
        hit += [("mean", ("dx", "df")), ("post mean", ("df",))]
    if gate != "none":
        hit += [("gate", ("df", "dw_post", "db_post"))]
    for drop, names in hit:
        over = worst(D, dtype, kind, gate, (drop,))
        for name in names:
            assert over[name] > 1, (drop, name, over[name])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_is_outside_where_it_is_zero(dtype):
    x, f, dy, dz, p, g = case(512, dtype, "sigmoid")
    ref, _ = ON.block(x, f, gate=g, sigmoid=True, res_scale=0.75, dy=dy, dz=dz, **p)
    for name, v in ON.normwise({k: 0 * v for k, v in ref.items()}, ref, HALF[dtype]).items():
        assert v > 1, name
