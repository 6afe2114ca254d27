"""GPU norms between two blocks (gate, scaled residual) vs the fp64 oracle, each result held to the bound that the
oracle derives for fp32 arithmetic and one rounding; and a whole layer of the new operators together."""

import sys

import numpy as np
import pytest
import torch

from oracle import norm as ON
from oracle import packed as OP
from synth.tensors import normal_tensor
from tests.helpers import dev_feat, host

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
FWD, BWD = ("y", "z"), ("dx", "df", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def make(n, D, dtype, gate, seed=0, affine=True):
    x, f, dy, dz = (normal_tensor((n, D), (seed, t), dtype) for t in range(4))
    rng = np.random.default_rng(seed)
    p = {}
    if affine:
        for name, mean in (("w_post", 1.0), ("b_post", 0.0), ("w_pre", 1.0), ("b_pre", 0.0)):
            p[name] = (mean + 0.3 * rng.normal(size=D)).astype(np.float32)
    if gate == "vector":
        p["gate"] = rng.normal(size=D).astype(np.float32)
    elif gate != "none":
        p["gate"] = normal_tensor((n, D), (seed, 9), dtype)
    return x, f, dy, dz, p


def check(name, x, r, b):
    x = np.asarray(x, dtype=np.float64)
    assert x.shape == r.shape and np.isfinite(x).all(), name
    over = np.abs(x - r) - b
    assert over.size == 0 or over.max() <= 0, (f"{name}: {int((over > 0).sum())}/{over.size} outside their bound, by "
                                               f"up to {over.max():.3e} (largest error {np.abs(x - r).max():.3e})")


def compare(gt, n, D, dtype, kind, gate, seed=0, affine=True, res_scale=0.75, eps=1e-5, inputs=None):
    say("norm", n, D, dtype, kind, gate)
    x, f, dy, dz, p = make(n, D, dtype, gate, seed, affine) if inputs is None else inputs
    dev = {k: dev_feat(v, dtype) if v.ndim == 2 else torch.from_numpy(v).cuda() for k, v in p.items()}
    X, F, dY, dZ = (dev_feat(v, dtype) for v in (x, f, dy, dz))
    args = dict(sigmoid=gate == "sigmoid", res_scale=res_scale, kind=kind, eps=eps, **dev)
    y, z, stats = gt.block_norm_fwd(X, F, **args)
    got = dict(zip(FWD + BWD, (y, z) + gt.block_norm_bwd(X, F, stats, dY, dZ, **args)))
    torch.cuda.synchronize()
    r, b = ON.block(x, f, sigmoid=gate == "sigmoid", res_scale=float(np.float32(res_scale)), layer=kind == "layer",
                    eps=float(np.float32(eps)), dy=dy, dz=dz, half=HALF[dtype], **p)
    for name in FWD + BWD:
        assert (got[name] is None) == (name not in r), name
        if name in r:
            check(name, host(got[name]), r[name], b[name])
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("gate", ["none", "vector", "rows", "sigmoid"])
def test_norms_gates_and_widths(gt, dtype, kind, gate):
    for n, D in ((1, 1), (3, 7), (33, 32), (70, 64), (65, 100), (9, 128), (17, 256), (130, 512), (5, 1000)):
        compare(gt, n, D, dtype, kind, gate, seed=n + D)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [513, 1024, 1536, 2048, 4096, 4100, 8191, 8192])
def test_wide_rows(gt, dtype, D):
    compare(gt, 6, D, dtype, "layer", "sigmoid", seed=D)
    compare(gt, 3, D, dtype, "rms", "vector", seed=D, affine=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 200, 1024])
def test_many_rows(gt, dtype, D):
    # more rows than one round of the grid
    a = compare(gt, 40_003 if D == 64 else 9_001, D, dtype, "layer", "vector", seed=1)
    b = compare(gt, 40_003 if D == 64 else 9_001, D, dtype, "layer", "vector", seed=1)
    assert all(a[k] is b[k] is None or torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [511, 512, 8192])
def test_rows_larger_than_the_last_level_cache(gt, dtype, D):
    # the rows' results are those of the same rows in two smaller calls
    n = (260 << 20) // (D * (2 if dtype == torch.bfloat16 else 4))
    g = torch.Generator(device="cuda").manual_seed(D)
    x, f, dy, dz, gate = (torch.randn(n, D, device="cuda", generator=g).to(dtype) for _ in range(5))
    w = torch.randn(D, device="cuda", generator=g)
    kw = dict(w_post=w, b_post=w, w_pre=w, b_pre=w, sigmoid=True)
    y, z, stats = gt.block_norm_fwd(x, f, gate=gate, **kw)
    grads = gt.block_norm_bwd(x, f, stats, dy, dz, gate=gate, **kw)
    h = n // 2
    for part in (slice(0, h), slice(h, n)):
        a = gt.block_norm_fwd(x[part], f[part], gate=gate[part], **kw)
        b = gt.block_norm_bwd(x[part], f[part], a[2], dy[part], dz[part], gate=gate[part], **kw)
        assert torch.equal(y[part], a[0]) and torch.equal(z[part], a[1]) and torch.equal(stats[part], a[2])
        assert all(torch.equal(grads[k][part], b[k]) for k in range(3))


def run(gt, x, f, dy, dz, p, dtype, kind, gate, res_scale=0.75, eps=1e-5):
    """The results of both calls by name, None left out."""
    dev = {k: dev_feat(v, dtype) if v.ndim == 2 else torch.from_numpy(v).cuda() for k, v in p.items()}
    X, F, dY, dZ = (dev_feat(v, dtype) for v in (x, f, dy, dz))
    args = dict(sigmoid=gate == "sigmoid", res_scale=res_scale, kind=kind, eps=eps, **dev)
    y, z, stats = gt.block_norm_fwd(X, F, **args)
    got = dict(zip(FWD + BWD, (y, z) + gt.block_norm_bwd(X, F, stats, dY, dZ, **args)))
    torch.cuda.synchronize()
    return {k: v for k, v in got.items() if v is not None}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("gate", ["none", "vector", "rows", "sigmoid"])
@pytest.mark.parametrize("D", [8, 40, 64, 100, 128, 256, 511, 512, 513, 1000, 1023, 1024, 1536, 2048, 2050, 4096, 4100,
                               8190, 8191, 8192])
def test_results_normwise(gt, dtype, kind, gate, D):
    # elementwise bounds of whole chains say little about gradients of wide rows: row by row in their size
    say("normwise", D, dtype, kind, gate)
    x, f, dy, dz, p = make(37 if D < 2048 else 9, D, dtype, gate, seed=D)
    got = run(gt, x, f, dy, dz, p, dtype, kind, gate)
    r, _ = ON.block(x, f, sigmoid=gate == "sigmoid", res_scale=0.75, layer=kind == "layer", eps=float(np.float32(1e-5)),
                    dy=dy, dz=dz, **p)
    assert set(got) == set(r)
    over = ON.normwise({k: host(v) for k, v in got.items()}, r, HALF[dtype])
    assert max(over.values()) <= 1, over


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,D", [(70_001, 24), (40_003, 64), (35_001, 200), (9_001, 1024), (9_001, 511), (2_100, 4096),
                                 (2_100, 8191)])
def test_every_row_counts_once(gt, dtype, n, D):
    # whole numbers, whose sums are exact in any order: a row lost or added twice in many rounds of the grid shows
    rng = np.random.default_rng(n + D)
    dy, dz = (rng.integers(-2, 3, size=(n, D)).astype(np.float32) for _ in range(2))
    x, f, _, _, p = make(n, D, dtype, "none", seed=D)
    p["w_pre"][:] = 0  # dz does not reach y: the gradient of y is dy
    got = run(gt, x, f, dy, dz, p, dtype, "layer", "none", res_scale=2.0)
    assert np.array_equal(host(got["db_pre"]), dz.sum(axis=0, dtype=np.float64))
    assert np.array_equal(host(got["db_post"]), dy.sum(axis=0, dtype=np.float64))
    assert np.array_equal(host(got["dx"]), 2.0 * dy)


def test_no_rows_and_views(gt):
    e = torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, device="cuda")
    y, z, st = gt.block_norm_fwd(e, e, w_post=w, gate=w)
    got = gt.block_norm_bwd(e, e, st, e, e, w_post=w, gate=w)
    torch.cuda.synchronize()
    assert y.shape == z.shape == (0, 64) and (got[2] == 0).all() and (got[3] == 0).all()
    # rows that start at any element
    x, f, dy, dz, _ = make(20, 64, "bf16", "none")
    odd = lambda v: torch.cat([torch.zeros(3, dtype=torch.bfloat16, device="cuda"),  # noqa: E731
                               dev_feat(v, "bf16").view(-1)])[3:].view(20, 64)
    a = gt.block_norm_fwd(odd(x), odd(f))
    b = gt.block_norm_fwd(dev_feat(x, "bf16"), dev_feat(f, "bf16"))
    ga = gt.block_norm_bwd(odd(x), odd(f), a[2], odd(dy), odd(dz))
    gb = gt.block_norm_bwd(dev_feat(x, "bf16"), dev_feat(f, "bf16"), b[2], dev_feat(dy, "bf16"), dev_feat(dz, "bf16"))
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(ga[0], gb[0]) and torch.equal(ga[1], gb[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_from_zero_and_flat_rows(gt, dtype):
    x, f, dy, dz, p = make(12, 96, dtype, "none")
    f[:6] = f[:6] + 64.0  # a mean far above the spread
    f[6] = 0.0  # no spread at all: eps decides
    if dtype == "bf16":
        from synth.tensors import bf16_round

        f = bf16_round(f)
    compare(gt, 12, 96, dtype, "layer", "none", inputs=(x, f, dy, dz, p), eps=1e-3)
    compare(gt, 12, 96, dtype, "rms", "none", inputs=(x, f, dy, dz, p), eps=1e-3)


def test_captured_norms_replay(gt):
    x, f, dy, dz, p = make(300, 256, "bf16", "sigmoid")
    dev = {k: dev_feat(v, "bf16") if v.ndim == 2 else torch.from_numpy(v).cuda() for k, v in p.items()}
    X, F, dY, dZ = (dev_feat(v, "bf16") for v in (x, f, dy, dz))

    def step():
        y, z, st = gt.block_norm_fwd(X, F, sigmoid=True, **dev)
        return (y, z) + gt.block_norm_bwd(X, F, st, dY, dZ, sigmoid=True, **dev)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for turn in range(4):
        X.copy_(dev_feat(normal_tensor(x.shape, (turn, 7), "bf16"), "bf16"))
        graph.replay()
        got = [v.clone() for v in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn


def test_a_layer_of_a_batch_of_graphs(gt):
    """One layer as a program runs it, fp32: projections, packed attention with the learned bias, and the norms around
    the block with a sigmoid gate; every parameter's and input's gradient against fp64 autograd of the formulas."""
    lens, H, d, B = [23, 40, 1, 26, 70], 4, 32, 9
    n, D = sum(lens), H * d
    rng = np.random.default_rng(8)
    p = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    ids = rng.integers(0, B, size=OP.pair_layout(lens, lens)[1]).astype(np.uint8)
    draw = lambda *s: rng.normal(size=s).astype(np.float32)  # noqa: E731
    val = dict(x=draw(n, D), h=draw(n, D), w_qkv=draw(D, 3 * D) / 12, w_o=draw(D, D) / 12, gate=draw(n, D),
               table=draw(B, H), w_post=1 + draw(D) / 5, b_post=draw(D) / 5, w_pre=1 + draw(D) / 5, b_pre=draw(D) / 5)
    dy, dz = draw(n, D), draw(n, D)

    t = {k: torch.from_numpy(v).cuda() for k, v in val.items()}
    plan, I = gt.packed_plan(p, heads=H), torch.from_numpy(ids).cuda()
    qkv = (t["h"] @ t["w_qkv"]).view(n, 3 * H, d)
    q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
    O, L = gt.packed_attn_fwd_bias(plan, q, k, v, t["table"], I)
    f = O.view(n, D) @ t["w_o"]
    norm = dict(w_post=t["w_post"], b_post=t["b_post"], w_pre=t["w_pre"], b_pre=t["b_pre"], gate=t["gate"],
                sigmoid=True, res_scale=0.8)
    y, z, st = gt.block_norm_fwd(t["x"], f, **norm)
    g = {}
    g["x"], df, g["gate"], g["w_post"], g["b_post"], g["w_pre"], g["b_pre"] = gt.block_norm_bwd(
        t["x"], f, st, torch.from_numpy(dy).cuda(), torch.from_numpy(dz).cuda(), **norm)
    g["w_o"] = O.view(n, D).t() @ df
    dO = (df @ t["w_o"].t()).view(n, H, d)
    dq, dk, dv, g["table"] = gt.packed_attn_bwd_bias(plan, q, k, v, t["table"], I, dO, L)
    dqkv = torch.cat([dq, dk, dv], 1).view(n, 3 * D)
    g["w_qkv"], g["h"] = t["h"].t() @ dqkv, dqkv @ t["w_qkv"].t()
    torch.cuda.synchronize()

    c = {k: torch.from_numpy(v).double().requires_grad_() for k, v in val.items()}
    qkv = (c["h"] @ c["w_qkv"]).view(n, 3, H, d)
    rows = []
    for s, m in enumerate(lens):
        sl = slice(p[s], p[s + 1])
        bias = c["table"][torch.from_numpy(OP.pair_buckets(ids, lens, lens, s))].permute(2, 0, 1)
        w = torch.softmax(torch.einsum("ihc,jhc->hij", qkv[sl, 0], qkv[sl, 1]) / np.sqrt(d) + bias, -1)
        rows.append(torch.einsum("hij,jhc->ihc", w, qkv[sl, 2]).reshape(m, D))
    f64 = torch.cat(rows) @ c["w_o"]
    ln = lambda a, w, b: torch.nn.functional.layer_norm(a, (D,), w, b, 1e-5)  # noqa: E731
    y64 = 0.8 * c["x"] + torch.sigmoid(c["gate"]) * ln(f64, c["w_post"], c["b_post"])
    z64 = ln(y64, c["w_pre"], c["b_pre"])
    ((y64 * torch.from_numpy(dy)).sum() + (z64 * torch.from_numpy(dz)).sum()).backward()
    # normwise, a chain of some ten fp32 stages of at most 384 terms each: 10 * 384 * 2^-24 = 2.3e-4
    near = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())  # noqa: E731
    for name, a, b in [("y", y, y64), ("z", z, z64)] + [("d" + k, g[k], c[k].grad) for k in val]:
        say(name, near(a, b.detach()))
        assert near(a, b.detach()) <= 2.3e-4, name
