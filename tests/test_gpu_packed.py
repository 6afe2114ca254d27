"""GPU packed-sequence attention and the learned bias by buckets vs the fp64 oracle.

Every result is held to the bound that the oracle derives for it (oracle/packed.py): fp32 dot products and sums in any
order, weights and score gradients rounded to the features' type where they multiply a row, results rounded once."""

import ctypes
import sys

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import packed as OP
from synth import make_workload
from synth.tensors import normal_tensor
from tests.helpers import assert_close, dev_csr, dev_feat, host

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
LOWEST = float(np.finfo(np.float32).min)


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def ptrs(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def make(lq, lk, H, Hkv, d, dtype, B=0, seed=0, extra=0):
    """Host inputs (fp32 values of the dtype) and, with B, a table and bytes of buckets (1 in 12 beyond it)."""
    shapes = ((sum(lq) + extra, H, d), (sum(lk) + extra, Hkv, d), (sum(lk) + extra, Hkv, d), (sum(lq) + extra, H, d))
    q, k, v, do = (normal_tensor(s, (seed, d, t), dtype) for t, s in enumerate(shapes))
    if not B:
        return q, k, v, do, None, None
    rng = np.random.default_rng(seed)
    _, n = OP.pair_layout(lq, lk)
    ids = rng.integers(0, B, size=n).astype(np.uint8)
    far = rng.random(n) < 1 / 12
    ids[far] = rng.integers(B, 256, size=int(far.sum()))
    return q, k, v, do, rng.normal(size=(B, H)).astype(np.float32), ids


def check(name, x, r, b):
    x = np.asarray(x, dtype=np.float64)
    fin = np.isfinite(r)
    assert np.array_equal(x[~fin], r[~fin]), f"{name}: infinite values differ"
    assert np.isfinite(x[fin]).all(), f"{name}: values that are not finite"
    over = np.abs(x[fin] - r[fin]) - b[fin]
    assert over.size == 0 or over.max() <= 0, (f"{name}: {int((over > 0).sum())}/{over.size} outside their bound, by "
                                               f"up to {over.max():.3e} (largest error {np.abs(x[fin] - r[fin]).max():.3e})")


def run(gt, lq, lk, H, Hkv, d, dtype, causal, inputs, scale):
    q, k, v, do, table, ids = inputs
    plan = gt.packed_plan(ptrs(lq), ptrs(lk), heads=H, kv_heads=Hkv, causal=causal)
    Q, K, V, dO = (dev_feat(x, dtype) for x in (q, k, v, do))
    if table is None:
        O, L = gt.packed_attn_fwd(plan, Q, K, V, scale)
        out = (O, L) + gt.packed_attn_bwd(plan, Q, K, V, O, dO, L, scale)
    else:
        T, I = torch.from_numpy(table).cuda(), torch.from_numpy(ids).cuda()
        O, L = gt.packed_attn_fwd_bias(plan, Q, K, V, T, I, scale)
        out = (O, L) + gt.packed_attn_bwd_bias(plan, Q, K, V, T, I, dO, L, scale)
    torch.cuda.synchronize()
    return out


def compare(gt, lq, lk, H, Hkv, d, dtype, causal, B=0, seed=0, scale=None, inputs=None, exact_d=False):
    say("packed", lq if len(lq) < 12 else len(lq), lk if len(lk) < 12 else "", H, Hkv, d, dtype, causal, B)
    inputs = make(lq, lk, H, Hkv, d, dtype, B, seed) if inputs is None else inputs
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out = run(gt, lq, lk, H, Hkv, d, dtype, causal, inputs, scale)
    q, k, v, do, table, ids = inputs
    r, b = OP.attn(ptrs(lq), ptrs(lk), q, k, v, np.float32(scale).astype(np.float64), causal, table, ids, do,
                   HALF[dtype], exact_d=exact_d or table is not None)
    for name, x in zip(("O", "LSE", "dQ", "dK", "dV", "dtable"), out):
        check(name, host(x), r[name], b[name])
    return out, r


SIZES = [
    ([1], [1]), ([5], [3]), ([0, 1, 2, 0], [3, 0, 1, 0]), ([31, 32, 33], [31, 32, 33]),
    ([63, 64, 65, 127, 128, 129], [129, 128, 127, 65, 64, 63]), ([257], [511]), ([1] * 9, [1, 7, 40, 64, 65, 200, 33, 0, 2]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B", [0, 7])
def test_sizes_where_tiles_end(gt, dtype, d, causal, B):
    for n, (lq, lk) in enumerate(SIZES):
        compare(gt, lq, lk, 2, 2, d, dtype, causal, B, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B", [0, 33])
def test_small_sequences_alone_and_in_large_batches(gt, dtype, d, causal, B):
    # none above 32 rows and keys: whole sequences a wavefront
    compare(gt, [31, 32, 1, 17, 0, 8, 32, 5], [32, 31, 5, 17, 3, 0, 32, 1], 4, 4, d, dtype, causal, B, seed=d)
    compare(gt, [7, 8, 1, 3], [32, 31, 5, 1], 8, 2, d, dtype, causal, B, seed=d + 1)
    # every list of tiles: more tiles than a batch may have whose small sequences go with the others
    lq, lk = [1, 30, 33, 50, 64, 65, 130, 2, 300, 20], [32, 30, 33, 70, 40, 65, 20, 100, 5, 300]
    compare(gt, lq * 4, lk * 4, 32, 32, d, dtype, causal, B, seed=d + 2)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (8, 2)])
@pytest.mark.parametrize("causal", [False, True])
def test_rows_of_few_keys_do_not_see_the_rounding_of_o(gt, d, H, Hkv, causal):
    # a row of one key has no score gradient at all, whatever a bf16 O says
    compare(gt, [33, 50, 64, 60], [33, 50, 64, 64], H, Hkv, d, "bf16", causal, seed=d + H, exact_d=True)
    compare(gt, [40] * 300, [2, 40, 50] * 100, H, Hkv, d, "bf16", causal, seed=d + H, exact_d=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 3), (4, 2), (4, 1), (8, 1), (16, 1), (32, 2)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B", [0, 64])
def test_grouped_heads(gt, dtype, H, Hkv, causal, B):
    compare(gt, [1, 2, 17, 40, 3], [70, 2, 17, 45, 1], H, Hkv, 32, dtype, causal, B, seed=H)
    compare(gt, [130], [150], H, Hkv, 64, dtype, causal, B, seed=H + 1)
    compare(gt, [2, 70, 30], [30, 33, 1100], H, Hkv, 128, dtype, causal, B, seed=H + 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
def test_long_and_many(gt, dtype, causal):
    compare(gt, [1200, 3, 800], [1200, 2500, 700], 2, 1, 64, dtype, causal)
    rng = np.random.default_rng(5)
    n = [int(x) for x in rng.integers(0, 30, size=300)]
    compare(gt, n, n, 4, 4, 32, dtype, causal, B=21)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_single_queries_over_long_keys(gt, dtype):
    # read-out tokens and single-token serving: few rows, long walks
    compare(gt, [1], [9001], 8, 8, 32, dtype, False)
    compare(gt, [1, 1, 2], [5003, 1, 4096], 16, 2, 128, dtype, True)
    compare(gt, [3], [6000], 4, 4, 64, dtype, True, B=5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [0, 5])
def test_long_walks_of_few_tiles_are_split(gt, dtype, B):
    # few rows beside many keys, few keys beside many rows, and both beside short sequences
    compare(gt, [100, 7], [4500, 9], 1, 1, 32, dtype, False, B)
    compare(gt, [4500, 3], [100, 200], 1, 1, 64, dtype, False, B)
    compare(gt, [60, 5], [3000, 2], 2, 1, 128, dtype, True, B)
    compare(gt, [2500, 40], [30, 2300], 2, 2, 32, dtype, True, B)


@pytest.mark.parametrize("dtype,d,H,causal,B", [("bf16", 32, 32, False, 0), ("bf16", 64, 32, False, 0),
                                                ("bf16", 128, 32, False, 0), ("f32", 32, 32, False, 0),
                                                ("f32", 128, 32, False, 0), ("bf16", 64, 32, False, 5),
                                                ("bf16", 128, 32, False, 64), ("f32", 64, 32, False, 64),
                                                ("bf16", 64, 32, True, 0), ("bf16", 64, 32, True, 21)])
def test_long_sequences_of_many_heads(gt, dtype, d, H, causal, B):
    """Enough long walks for the largest tiles; two heads against a plain implementation in 64 bits on the GPU."""
    lens = [2333, 2304]
    say("large", dtype, d, H, causal, B)
    p, scale = ptrs(lens), 1.0 / np.sqrt(d)
    q, k, v, do, table, ids = make(lens, lens, H, H, d, dtype, B, seed=d + B)
    plan = gt.packed_plan(p, heads=H, causal=causal)
    assert causal or plan.c.layout[2 * 4 + 1] > 0 and plan.c.layout[2 * 8 + 1] > 0  # tiles of 256 rows and keys
    out = run(gt, lens, lens, H, H, d, dtype, causal, (q, k, v, do, table, ids), scale)
    half, u, scale = HALF[dtype], 2.0 ** -24, float(np.float32(scale))
    dt = torch.zeros(B, dtype=torch.float64, device="cuda"), torch.zeros(B, dtype=torch.float64, device="cuda")
    for h in (0, H - 1):
        for x in dt:
            x.zero_()
        for s, n in enumerate(lens):
            sl = slice(int(p[s]), int(p[s + 1]))
            Q, K, V, G = (torch.from_numpy(x[sl, h]).cuda().double() for x in (q, k, v, do))
            sc = scale * (Q @ K.t())
            if B:
                id_ = torch.from_numpy(OP.pair_buckets(ids, lens, lens, s)).cuda()
                T = torch.cat([torch.from_numpy(table[:, h]).cuda().double(),
                               torch.full((256 - B,), -np.inf, dtype=torch.float64, device="cuda")])
                sc = sc + T[id_]
            if causal:
                sc = sc.masked_fill(torch.ones_like(sc, dtype=torch.bool).triu(1), -np.inf)
            P = torch.softmax(sc, -1)
            dP = G @ V.t()
            D = (P * dP).sum(-1, keepdim=True)
            dS = P * (dP - D)
            # scores, weights and dP in fp32 (d terms of at most 8 in all); sums of n terms; D from a bf16 O without a bias
            w = 4 * (d + 8) * u * 8 + 2 * n * u
            e_o = (half + w) * (P @ V.abs()) + half * (P @ V).abs()
            e_d = (G.abs() * e_o).sum(-1, keepdim=True) if not B else w * (P * dP.abs()).sum(-1, keepdim=True)
            e_ds = w * dS.abs() + P * (e_d + d * u * (G.abs() @ V.abs().t()))
            refs = [("O", out[0], P @ V, e_o), ("LSE", out[1], torch.logsumexp(sc, -1), torch.full((n,), w).cuda()),
                    ("dQ", out[2], scale * dS @ K, scale * (e_ds + (half + w) * dS.abs()) @ K.abs()),
                    ("dK", out[3], scale * dS.t() @ Q, scale * (e_ds + (half + w) * dS.abs()).t() @ Q.abs()),
                    ("dV", out[4], P.t() @ G, ((half + w) * P).t() @ G.abs())]
            for name, x, r, e in refs:
                err = (x[sl, h].double() - r).abs() - (e + 2 * half * r.abs())
                assert float(err.max()) <= 0, f"{name} head {h} sequence {s}: outside its bound by {float(err.max()):.2e}"
            if B:
                dt[0].add_(torch.bincount(id_.flatten(), weights=dS.flatten(), minlength=256)[:B])
                dt[1].add_(torch.bincount(id_.flatten(), weights=(e_ds + 4096 * u * dS.abs()).flatten(), minlength=256)[:B])
        if B:
            assert float(((out[5][:, h].double() - dt[0]).abs() - dt[1]).max()) <= 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [0, 9])
@pytest.mark.parametrize("lq,lk,H,Hkv,d,causal", [
    ([1200, 3, 800], [1200, 2500, 700], 2, 1, 64, False), ([1200, 3, 800], [1200, 2500, 700], 2, 1, 64, True),
    ([1], [9001], 8, 8, 32, False), ([1, 2], [5003, 4096], 16, 2, 128, True), ([100, 7], [4500, 9], 1, 1, 32, False),
    ([4500, 3], [100, 200], 1, 1, 64, False), ([700], [2500], 4, 4, 128, True), ([300] * 24, [300] * 24, 8, 8, 32, True),
    ([45] * 200, [45] * 200, 4, 4, 64, False), ([24] * 400, [24] * 400, 4, 4, 32, False), ([60] * 150, [60] * 150, 8, 8, 32, False)])
def test_results_normwise(gt, dtype, B, lq, lk, H, Hkv, d, causal):
    # whole arrays in their size, over long, split, mid-sized and small sequences (the elementwise bounds add the terms of
    # a row as absolute values)
    say("normwise", len(lq), lq[0], lk[0], H, Hkv, d, dtype, causal, B)
    inputs = make(lq, lk, H, Hkv, d, dtype, B, seed=d + B)
    scale = 1.0 / np.sqrt(d)
    out = run(gt, lq, lk, H, Hkv, d, dtype, causal, inputs, scale)
    q, k, v, do, table, ids = inputs
    r, _ = OP.attn(ptrs(lq), ptrs(lk), q, k, v, np.float32(scale).astype(np.float64), causal, table, ids, do, HALF[dtype])
    got = {name: host(x) for name, x in zip(("O", "LSE", "dQ", "dK", "dV"), out)}
    over = OP.normwise(got, r, HALF[dtype], max(max(lk), max(lq) * (H // Hkv)))
    say("   ", over)
    assert len(over) == 4 and max(over.values()) <= 1, over


@pytest.mark.parametrize("dtype,d,causal,B", [("bf16", 32, False, 0), ("bf16", 64, False, 0), ("bf16", 128, False, 0),
                                              ("f32", 32, False, 0), ("f32", 64, True, 0), ("f32", 128, False, 0),
                                              ("bf16", 64, False, 5), ("bf16", 128, True, 64), ("f32", 64, False, 64),
                                              ("bf16", 64, True, 0)])
def test_long_sequences_of_many_heads_normwise(gt, dtype, d, causal, B):
    """The largest tiles: every head's results as whole arrays, against a plain implementation in 64 bits on the GPU."""
    lens, H = [2333, 2304], 32
    say("large, normwise", dtype, d, causal, B)
    p, scale = ptrs(lens), float(np.float32(1.0 / np.sqrt(d)))
    inputs = make(lens, lens, H, H, d, dtype, B, seed=d + B)
    out = run(gt, lens, lens, H, H, d, dtype, causal, inputs, scale)
    table, ids = inputs[4:]
    for h in (0, 7, H - 1):
        ref = [torch.empty(sum(lens), d, dtype=torch.float64, device="cuda") for _ in range(4)]
        for s, n in enumerate(lens):
            sl = slice(int(p[s]), int(p[s + 1]))
            Q, K, V, G = (torch.from_numpy(x[sl, h]).cuda().double() for x in inputs[:4])
            sc = scale * (Q @ K.t())
            if B:
                more = torch.full((256,), -np.inf, dtype=torch.float64, device="cuda")
                more[:B] = torch.from_numpy(table[:, h]).cuda()
                sc = sc + more[torch.from_numpy(OP.pair_buckets(ids, lens, lens, s)).cuda()]
            if causal:
                sc = sc.masked_fill(torch.ones_like(sc, dtype=torch.bool).triu(1), -np.inf)
            # a causal row's only keys may all lie beyond the table
            P = torch.nan_to_num(torch.softmax(sc, -1))
            dP = G @ V.t()
            dS = P * (dP - (P * dP).sum(-1, keepdim=True))
            for x, r in zip(ref, (P @ V, scale * dS @ K, scale * dS.t() @ Q, P.t() @ G)):
                x[sl] = r
        got = dict(zip(("O", "dQ", "dK", "dV"), (host(out[k])[:, h:h + 1] for k in (0, 2, 3, 4))))
        over = OP.normwise(got, dict(zip(got, (x.cpu().numpy()[:, None] for x in ref))), HALF[dtype], max(lens))
        say("   ", over)
        assert max(over.values()) <= 1, (h, over)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.5])
def test_any_scale(gt, dtype, scale):
    compare(gt, [70], [90], 2, 2, 32, dtype, True, scale=scale)
    compare(gt, [70], [90], 2, 2, 32, dtype, True, B=4, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_that_leave_rows_empty(gt, dtype):
    lq, lk, H, B = [50, 40], [50, 70], 2, 6
    inputs = list(make(lq, lk, H, H, 32, dtype, B, seed=9))
    table, ids = inputs[4], inputs[5]
    at, _ = OP.pair_layout(lq, lk)
    ids[at[0] + 3 * 64:at[0] + 5 * 64] = 255  # two queries without any pair
    ids[at[1]:] = np.where(np.arange(len(ids) - at[1]) % 80 < 33, 200, ids[at[1]:])  # the first 33 keys of every row
    table[2] = -np.inf  # a bucket that masks
    table[3, 0] = LOWEST  # and one that all but does
    out, r = compare(gt, lq, lk, H, H, 32, dtype, False, B, inputs=inputs)
    assert np.isneginf(host(out[1])[3:5]).all() and (host(out[0])[3:5] == 0).all() and (host(out[2])[3:5] == 0).all()
    assert (host(out[5])[2] == 0).all()
    # every pair masked, of every sequence
    ids[:] = B
    out, _ = compare(gt, lq, lk, H, H, 32, dtype, True, B, inputs=inputs)
    assert all((host(x) == 0).all() for n, x in enumerate(out) if n != 1) and np.isneginf(host(out[1])).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("level", [LOWEST, -1e30, -1e9, 1e6])
def test_a_bias_that_swamps_the_scores_still_averages(gt, dtype, level):
    # beside a bias this large an fp32 score holds nothing of <q, k> (or of log n): every pair weighs 1 / n
    lq, lk, H = [37], [90], 2
    q, k, v, do, _, _ = make(lq, lk, H, H, 32, dtype)
    q, k = q * 0, k * 0
    table = np.full((1, H), level, dtype=np.float32)
    ids = np.zeros(OP.pair_layout(lq, lk)[1], dtype=np.uint8)
    out = run(gt, lq, lk, H, H, 32, dtype, False, (q, k, v, do, table, ids), 0.2)
    mean = v.astype(np.float64).mean(axis=0)
    tol = 2 * HALF[dtype] + 128 * 2.0 ** -24
    np.testing.assert_allclose(host(out[0]), np.broadcast_to(mean, out[0].shape), atol=tol * np.abs(v).max())
    # dV_j = sum_i dO_i / n: half a step of each rounded weight and of the result, on the sum of |dO|
    dv = np.broadcast_to(do.astype(np.float64).sum(axis=0) / 90, out[4].shape)
    np.testing.assert_allclose(host(out[4]), dv, atol=2 * tol * np.abs(do).sum(axis=0).max() / 90)


def test_a_query_of_nan_stays_in_its_sequence_and_ends_do_not_leak(gt):
    # sequences 0 and 2 hold infinities and NaN everywhere: sequence 1, ragged against every tile, does not see them
    for dtype in ("bf16", "f32"):
        for lens in ([33, 45, 70], [200, 135, 9]):
            for B in (0, 5):
                say("neighbours", dtype, lens, B)
                inputs = list(make(lens, lens, 2, 2, 64, dtype, B, seed=3))
                p = ptrs(lens)
                clean = [x if x is None else x.copy() for x in inputs]
                for x in inputs[:4]:
                    x[:p[1]], x[p[2]:] = np.nan, np.inf
                a = run(gt, lens, lens, 2, 2, 64, dtype, True, inputs, 0.125)
                b = run(gt, lens, lens, 2, 2, 64, dtype, True, clean, 0.125)
                for x, y in zip(a[:5], b[:5]):
                    assert torch.equal(x[p[1]:p[2]], y[p[1]:p[2]])


@pytest.mark.parametrize("B", [0, 9])
def test_slices_of_a_fused_projection(gt, B):
    lq = [70, 3, 129]
    for dtype in ("bf16", "f32"):
        H, Hkv, d = 4, 2, 32
        q, k, v, do, table, ids = inputs = make(lq, lq, H, Hkv, d, dtype, B)
        want = run(gt, lq, lq, H, Hkv, d, dtype, True, inputs, 0.2)
        wide = torch.full((sum(lq), H + 2 * Hkv + 1, d), float("nan"), dtype=want[0].dtype, device="cuda")
        wide[:, :H], wide[:, H:H + Hkv], wide[:, H + Hkv:-1] = (dev_feat(x, dtype) for x in (q, k, v))
        Q, K, V = wide[:, :H], wide[:, H:H + Hkv], wide[:, H + Hkv:-1]
        plan, dO = gt.packed_plan(ptrs(lq), heads=H, kv_heads=Hkv, causal=True), dev_feat(do, dtype)
        if B:
            T, I = torch.from_numpy(table).cuda(), torch.from_numpy(ids).cuda()
            O, L = gt.packed_attn_fwd_bias(plan, Q, K, V, T, I, 0.2)
            got = (O, L) + gt.packed_attn_bwd_bias(plan, Q, K, V, T, I, dO, L, 0.2)
        else:
            O, L = gt.packed_attn_fwd(plan, Q, K, V, 0.2)
            got = (O, L) + gt.packed_attn_bwd(plan, Q, K, V, O, dO, L, 0.2)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("B", [0, 9])
def test_rows_behind_the_last_sequence(gt, B):
    lq, lk, H, d = [40, 33], [60, 5], 2, 32
    q, k, v, do, table, ids = make(lq, lk, H, H, d, "bf16", B, extra=7)
    for x in (q, k, v, do):
        x[-7:] = np.nan  # not read
    plan = gt.packed_plan(ptrs(lq), ptrs(lk), heads=H)
    Q, K, V, dO = (dev_feat(x, "bf16") for x in (q, k, v, do))
    if B:
        T, I = torch.from_numpy(table).cuda(), torch.from_numpy(ids).cuda()
        O, L = gt.packed_attn_fwd_bias(plan, Q, K, V, T, I)
        out = (O, L) + gt.packed_attn_bwd_bias(plan, Q, K, V, T, I, dO, L)
    else:
        O, L = gt.packed_attn_fwd(plan, Q, K, V)
        out = (O, L) + gt.packed_attn_bwd(plan, Q, K, V, O, dO, L)
    torch.cuda.synchronize()
    for n, x in enumerate(out[:5]):
        assert torch.isfinite(x[:-7].float()).all()
        assert (x[-7:] == (-np.inf if n == 1 else 0)).all()
    # the C call leaves such rows as they were
    lib, code = gt.load_library(), gt.GT_BF16
    O, L = torch.full_like(Q, 5.0), torch.full_like(out[1], 5.0)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    assert lib.gt_packed_attn_fwd(ctypes.byref(plan.c), d, code, Q.data_ptr(), H * d, K.data_ptr(), H * d, V.data_ptr(),
                                  H * d, 0.1, O.data_ptr(), L.data_ptr(), ws.data_ptr(), ws.numel(),
                                  torch.cuda.current_stream().cuda_stream) == gt.GT_OK
    dQ, dK, dV = torch.full_like(Q, 5.0), torch.full_like(K, 5.0), torch.full_like(V, 5.0)
    assert lib.gt_packed_attn_bwd(ctypes.byref(plan.c), d, code, Q.data_ptr(), H * d, K.data_ptr(), H * d, V.data_ptr(),
                                  H * d, O.data_ptr(), dO.data_ptr(), L.data_ptr(), 0.1, dQ.data_ptr(), dK.data_ptr(),
                                  dV.data_ptr(), ws.data_ptr(), ws.numel(),
                                  torch.cuda.current_stream().cuda_stream) == gt.GT_OK
    torch.cuda.synchronize()
    for x in (O, L, dQ, dK, dV):
        assert (x[-7:] == 5).all() and torch.isfinite(x.float()).all()


def test_no_sequences(gt):
    f = torch.zeros(0, 2, 32, dtype=torch.bfloat16, device="cuda")
    plan = gt.packed_plan([0], heads=2)
    O, L = gt.packed_attn_fwd(plan, f, f, f)
    out = gt.packed_attn_bwd(plan, f, f, f, O, f, L)
    T, I = torch.ones(3, 2, device="cuda"), torch.zeros(0, dtype=torch.uint8, device="cuda")
    O, L = gt.packed_attn_fwd_bias(plan, f, f, f, T, I)
    out = gt.packed_attn_bwd_bias(plan, f, f, f, T, I, f, L)
    torch.cuda.synchronize()
    assert O.shape == f.shape and (out[3] == 0).all()
    # keys that no query reads: their gradients are zeros, not left over
    k = torch.ones(5, 2, 32, dtype=torch.bfloat16, device="cuda")
    plan = gt.packed_plan([0, 0], [0, 5], heads=2)
    _, dk, dv = gt.packed_attn_bwd(plan, f, k, k, f, f, L[:0])
    torch.cuda.synchronize()
    assert (dk == 0).all() and (dv == 0).all()


def test_same_results_again_and_on_another_stream(gt):
    lq = [300, 20, 1, 77]
    for dtype in ("bf16", "f32"):
        for B in (0, 11):
            inputs = make(lq, lq, 4, 2, 64, dtype, B)
            a = run(gt, lq, lq, 4, 2, 64, dtype, True, inputs, 0.1)
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                b = run(gt, lq, lq, 4, 2, 64, dtype, True, inputs, 0.1)
            assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("mode", ["forward", "backward", "bias forward", "bias backward"])
def test_a_plan_dropped_while_another_stream_reads_it(gt, mode):
    # the memory of a plan's work list is not handed out again while a call on another stream than the plan's may read it
    lq = [70, 5, 200]
    q, k, v, do, table, ids = make(lq, lq, 2, 2, 32, "bf16", 4)
    Q, K, V, dO = (dev_feat(x, "bf16") for x in (q, k, v, do))
    T, I = torch.from_numpy(table).cuda(), torch.from_numpy(ids).cuda()
    plan = gt.packed_plan(ptrs(lq), heads=2)
    O, L = gt.packed_attn_fwd(plan, Q, K, V)
    Ob, Lb = gt.packed_attn_fwd_bias(plan, Q, K, V, T, I)
    call = {"forward": lambda p: gt.packed_attn_fwd(p, Q, K, V),
            "backward": lambda p: gt.packed_attn_bwd(p, Q, K, V, O, dO, L),
            "bias forward": lambda p: gt.packed_attn_fwd_bias(p, Q, K, V, T, I),
            "bias backward": lambda p: gt.packed_attn_bwd_bias(p, Q, K, V, T, I, dO, Lb)}[mode]
    want = call(plan)
    busy = torch.zeros(8192, 8192, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        busy @ busy
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(300):
            busy @ busy
        got = call(plan)
    at, n = plan.items.data_ptr(), plan.items.numel()
    del plan
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(64)]
    assert not side.query(), "the stream ran empty: this says nothing"
    assert all(x.data_ptr() != at for x in blocks)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B", [0, 9])
def test_sequences_without_keys_or_queries_beside_others(gt, dtype, d, causal, B):
    # more rows (or keys) than a small sequence's, in every list of tiles, with nothing to walk
    compare(gt, [100, 0, 70, 300, 0, 40, 1], [0, 100, 50, 0, 300, 0, 0], 2, 2, d, dtype, causal, B, seed=d)
    compare(gt, [20, 0, 70, 300, 50] * 40, [0, 40, 50, 0, 60] * 40, 16, 4, d, dtype, causal, B, seed=d + 1)
    compare(gt, [3000, 0], [0, 2600], 1, 1, d, dtype, causal, B, seed=d + 2)


def test_captured_step_replays(gt):
    lq, H, d, B = [150, 30, 33], 4, 32, 6
    q, k, v, do, table, ids = make(lq, lq, H, 2, d, "bf16", B)
    plan = gt.packed_plan(ptrs(lq), heads=H, kv_heads=2)
    Q, K, V, dO = (dev_feat(x, "bf16") for x in (q, k, v, do))
    T, I = torch.from_numpy(table).cuda(), torch.from_numpy(ids).cuda()

    def step():
        O, L = gt.packed_attn_fwd_bias(plan, Q, K, V, T, I)
        return (O, L) + gt.packed_attn_bwd_bias(plan, Q, K, V, T, I, dO, L)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for turn in range(4):
        Q.copy_(dev_feat(normal_tensor(q.shape, (turn, 1), "bf16"), "bf16"))
        graph.replay()
        got = [x.clone() for x in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), turn


@pytest.mark.parametrize("H", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("nnz,B", [(0, 3), (1, 1), (37, 5), (1000, 64), (70001, 21)])
def test_edge_bias_and_its_gradient(gt, H, nnz, B):
    say("edges", nnz, H, B)
    rng = np.random.default_rng(nnz + H)
    table, ids = rng.normal(size=(B, H)).astype(np.float32), rng.integers(0, B + 1, size=nnz).astype(np.uint8)
    grad = rng.normal(size=(nnz, H)).astype(np.float32)
    ids[rng.random(nnz) < 0.02] = 255
    T, I, G = torch.from_numpy(table).cuda(), torch.from_numpy(ids).cuda(), torch.from_numpy(grad).cuda()
    bias, dt = gt.bucket_bias_fwd(T, I), gt.bucket_bias_bwd(I, G, B)
    again = gt.bucket_bias_bwd(I, G, B)
    torch.cuda.synchronize()
    assert np.array_equal(bias.cpu().numpy(), OP.bucket_bias(table, ids))
    ref = OP.bucket_bias_grad(ids, grad, B)
    # chains of at most 4,096 additions
    bound = (min(nnz, 4096) + 4) * 2.0 ** -24 * OP.bucket_bias_grad(ids, np.abs(grad), B)
    check("dtable", dt.cpu().numpy(), ref, bound)
    assert torch.equal(dt, again)


@pytest.mark.parametrize("H,nnz", [(16, 4_300_003), (1, 68_000_001)])
def test_edge_bias_larger_than_the_last_level_cache(gt, H, nnz):
    table = torch.randn(21, H, device="cuda")
    ids = torch.randint(0, 21, (nnz,), dtype=torch.uint8, device="cuda")
    bias = gt.bucket_bias_fwd(table, ids)
    assert torch.equal(bias, table[ids.long()])
    dt = gt.bucket_bias_bwd(ids, bias, 21)
    # every value of a bucket is the table's: the sum is the count times it, chains of at most 4 nnz / 65,536 + 2^12
    n = torch.bincount(ids.long(), minlength=21).double()[:, None]
    ref = n * table.double()
    assert ((dt - ref).abs() <= (4 * nnz / 65536 + 4096) * 2.0 ** -24 * ref.abs()).all()


@pytest.mark.parametrize("H,nnz,B", [(16, 4_300_003, 21), (8, 9_000_001, 64), (1, 68_000_001, 21), (2, 3_000_017, 1)])
def test_every_edge_counts_once(gt, H, nnz, B):
    # whole numbers whose sums stay below 2^24, exact in any order: an edge lost or added twice in many rounds of the grid
    # shows
    g = torch.Generator(device="cuda").manual_seed(nnz)
    ids = torch.randint(0, B + 1, (nnz,), dtype=torch.uint8, device="cuda", generator=g)  # one bucket more than the table's
    grad = torch.randint(-2, 4, (nnz, H), device="cuda", generator=g, dtype=torch.int8)
    dt = gt.bucket_bias_bwd(ids, grad.float(), B)
    want = torch.stack([torch.bincount(ids, weights=grad[:, h].double(), minlength=B)[:B] for h in range(H)], 1)
    most = torch.bincount(ids, minlength=B)[:B].max() * 3
    assert most < 2 ** 24 and torch.equal(dt.double(), want)


def test_edge_bias_on_views_that_start_anywhere(gt):
    rng = np.random.default_rng(1)
    ids = torch.from_numpy(rng.integers(0, 5, size=1003).astype(np.uint8)).cuda()[3:]
    table = torch.randn(5, 4, device="cuda")
    grad = torch.randn(4 * 1000 + 1, device="cuda")[1:].view(1000, 4)
    bias, dt = gt.bucket_bias_fwd(table, ids), gt.bucket_bias_bwd(ids, grad, 5)
    torch.cuda.synchronize()
    assert torch.equal(bias, table[ids.long()])
    ref = OP.bucket_bias_grad(ids.cpu().numpy(), grad.cpu().numpy(), 5)
    np.testing.assert_allclose(dt.cpu().numpy(), ref, atol=1004 * 2.0 ** -24 * float(grad.abs().sum(0).max()))


def test_sparse_layer_with_a_learned_bias(gt):
    # the learned bias feeding the sparse layer's bias calls, on a plan with dense tiles, forward and backward
    w = make_workload("c5", 0.02)
    g, B = w.graph, 21
    q, k, v, do = w.tensors()
    scale = 1.0 / np.sqrt(w.dim)
    rng = np.random.default_rng(4)
    table, ids = rng.normal(size=(B, w.heads)).astype(np.float32), rng.integers(0, B, size=g.nnz).astype(np.uint8)
    rp, cl = dev_csr(g.rowptr, g.col)
    plan = gt.build_tiles(rp, cl, 128, 10000, edge_positions=True)
    Q, K, V, dO = (dev_feat(x, "bf16") for x in (q, k, v, do))
    T, I = torch.from_numpy(table).cuda(), torch.from_numpy(ids).cuda()
    bias = gt.bucket_bias_fwd(T, I)
    O, L = gt.sparse_attn_fwd_bias(plan, Q, K, V, bias, scale)
    dQ, dK, dV, dB = gt.sparse_attn_bwd_bias(plan, gt.edge_map(plan), Q, K, V, bias, dO, L, scale)
    dT = gt.bucket_bias_bwd(I, dB, B)
    torch.cuda.synchronize()
    b64 = OP.bucket_bias(table, ids)
    O_ref, _ = OA.sparse_attn_fwd(g.rowptr, g.col, q, k, v, scale, bias=b64)
    ref = OA.sparse_attn_bwd(g.rowptr, g.col, q, k, v, do, scale, bias=b64)
    for name, x, r in zip(("O", "dQ", "dK", "dV"), (O, dQ, dK, dV), (O_ref, *ref[:3])):
        assert_close(host(x), r, "bf16", name)
    # the edges' own tolerance (bf16, 2e-2 + 1e-2 |r|), summed over each bucket's edges
    bound = OP.bucket_bias_grad(ids, 2e-2 + 1e-2 * np.abs(ref[3]), B)
    check("dtable", dT.cpu().numpy(), OP.bucket_bias_grad(ids, ref[3], B), bound)
