"""GPU packed attention, learned bias and norms where offsets pass 32 bits, at the largest strides and head counts, and
replayed from captured graphs."""

import sys

import numpy as np
import pytest
import torch

from oracle import packed as OP
from synth.tensors import normal_tensor
from tests.helpers import dev_feat, host
from tests.test_gpu_packed import HALF, check, compare, make, ptrs, run

pytestmark = pytest.mark.gpu

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [0, 5])
def test_widest_strides(gt, dtype, B):
    # nodes 2^23 - 8 elements apart, the arrays' ends 2 to 10 GB from their starts
    lens, H, Hkv, d, ld = [70, 20, 200], 4, 2, 32, (1 << 23) - 8
    say("strides", dtype, B)
    inputs = make(lens, lens, H, Hkv, d, dtype, B, seed=1)
    want = run(gt, lens, lens, H, Hkv, d, dtype, True, inputs, 0.2)
    q, k, v, do, table, ids = inputs
    n = sum(lens)
    wide = torch.empty(n * ld, dtype=DTYPE[dtype], device="cuda").view(n, ld)
    at = [wide[:, o:o + h * d].unflatten(1, (h, d)) for o, h in ((ld - H * d, H), (0, Hkv), (1 << 22, Hkv))]
    for x, y in zip(at, (q, k, v)):
        x.copy_(dev_feat(y, dtype))
    plan, dO = gt.packed_plan(ptrs(lens), heads=H, kv_heads=Hkv, causal=True), dev_feat(do, dtype)
    if B:
        T, I = torch.from_numpy(table).cuda(), torch.from_numpy(ids).cuda()
        O, L = gt.packed_attn_fwd_bias(plan, *at, T, I, 0.2)
        got = (O, L) + gt.packed_attn_bwd_bias(plan, *at, T, I, dO, L, 0.2)
    else:
        O, L = gt.packed_attn_fwd(plan, *at, 0.2)
        got = (O, L) + gt.packed_attn_bwd(plan, *at, O, dO, L, 0.2)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_buckets_beyond_four_gigabytes(gt, dtype):
    # one sequence of 66,000 queries and keys: 4.4 GB of buckets; every result normwise against 64 bits, row by row
    n, B, d = 66_001, 12, 32
    say("buckets", dtype)
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v, do = (torch.randn(n, 1, d, device="cuda", generator=g).to(DTYPE[dtype]) for _ in range(4))
    plan = gt.packed_plan([0, n], heads=1)
    wide = (n + 15) // 16 * 16
    assert plan.pair_bytes == n * wide > 1 << 32
    ids = torch.randint(0, B + 1, (plan.pair_bytes,), dtype=torch.uint8, device="cuda", generator=g)
    table = torch.randn(B, 1, device="cuda", generator=g)
    scale = float(np.float32(1 / np.sqrt(d)))
    O, L = gt.packed_attn_fwd_bias(plan, q, k, v, table, ids, scale)
    dQ, dK, dV, dT = gt.packed_attn_bwd_bias(plan, q, k, v, table, ids, do, L, scale)
    Q, K, V, G = (x[:, 0].double() for x in (q, k, v, do))
    more = torch.full((256,), -np.inf, dtype=torch.float64, device="cuda")
    more[:B] = table[:, 0]
    ref = {x: torch.zeros(n, d, dtype=torch.float64, device="cuda") for x in ("O", "dQ", "dK", "dV")}
    lse, dt, size = torch.empty(n, dtype=torch.float64, device="cuda"), torch.zeros(256, dtype=torch.float64, device="cuda"), 0.0
    rows = ids.view(n, wide)[:, :n]
    for a in range(0, n, 2000):
        sl = slice(a, min(n, a + 2000))
        id_ = rows[sl].int()
        sc = scale * (Q[sl] @ K.t()) + more[id_]
        lse[sl] = torch.logsumexp(sc, -1)
        P = torch.exp(sc - lse[sl, None])
        dP = G[sl] @ V.t()
        dS = P * (dP - (P * dP).sum(-1, keepdim=True))
        ref["O"][sl], ref["dQ"][sl] = P @ V, scale * dS @ K
        ref["dK"] += scale * dS.t() @ Q[sl]
        ref["dV"] += P.t() @ G[sl]
        dt += torch.bincount(id_.flatten(), weights=dS.flatten(), minlength=256)
        size += float(dS.abs().sum())
    got = dict(zip(("O", "dQ", "dK", "dV"), (host(x) for x in (O, dQ, dK, dV))))
    over = OP.normwise(got, {x: y.cpu().numpy()[:, None] for x, y in ref.items()}, HALF[dtype], n)
    say("   ", over, float((dT[:, 0].double() - dt[:B]).abs().max()), size)
    assert max(over.values()) <= 1, over
    # scores of at most 16 in fp32 (d + 4 terms), a sum of 66,001 weights in chains of at most 2,100
    assert float((L[:, 0].double() - lse).abs().max()) <= (36 * 16 + 2100) * 2.0 ** -24
    # a weight's error, and chains of at most 66,001 / 32 * 16 additions in a lane's column
    assert float((dT[:, 0].double() - dt[:B]).abs().max()) <= 33_000 * 2.0 ** -24 * size


@pytest.mark.parametrize("B", [0, 7])
def test_features_beyond_2_to_31_elements(gt, B):
    # 20,000 sequences of 30 and a last one of 500, 32 heads of 128: 2.46e9 elements an array; the last ones against fp64
    lens, H, d = [30] * 20_000 + [500, 31], 32, 128
    say("elements", B)
    p = ptrs(lens)
    n = int(p[-1])
    assert n * H * d > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v, do = (torch.empty(n, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(4))
    plan = gt.packed_plan(p, heads=H)
    if B:
        ids = torch.randint(0, B + 1, (plan.pair_bytes,), dtype=torch.uint8, device="cuda", generator=g)
        table = torch.randn(B, H, device="cuda", generator=g)
        O, L = gt.packed_attn_fwd_bias(plan, q, k, v, table, ids)
        grads = gt.packed_attn_bwd_bias(plan, q, k, v, table, ids, do, L)
    else:
        O, L = gt.packed_attn_fwd(plan, q, k, v)
        grads = gt.packed_attn_bwd(plan, q, k, v, O, do, L)
    last, heads = slice(int(p[-4]), n), slice(H - 2, H)
    lq = lens[-3:]
    cut = lambda x: x[last, heads].double().cpu().numpy()  # noqa: E731
    tail = ids[-OP.pair_layout(lq, lq)[1]:].cpu().numpy() if B else None
    r, b = OP.attn(ptrs(lq), ptrs(lq), cut(q), cut(k), cut(v), float(np.float32(1 / np.sqrt(d))), False,
                   table[:, heads].cpu().numpy() if B else None, tail, cut(do), HALF["bf16"], exact_d=B > 0)
    for name, x in zip(("O", "LSE", "dQ", "dK", "dV"), (O, L) + tuple(grads)):
        check(name, cut(x), r[name], b[name])


def test_norms_beyond_2_to_31_elements(gt):
    n, D = 270_000, 8192
    say("norms")
    assert n * D > 1 << 31
    x = torch.empty(n, D, dtype=torch.bfloat16, device="cuda")
    for a in range(0, n, 30_000):
        x[a:a + 30_000].normal_()
    f = x.flip(0)
    w = torch.randn(D, device="cuda")
    kw = dict(w_post=w, b_post=w, w_pre=w, b_pre=w, gate=w)
    y, z, stats = gt.block_norm_fwd(x, f, **kw)
    grads = gt.block_norm_bwd(x, f, stats, f, x, **kw)
    t = slice(n - 700, n)
    a = gt.block_norm_fwd(x[t], f[t], **kw)
    b = gt.block_norm_bwd(x[t], f[t], a[2], f[t], x[t], **kw)
    assert torch.equal(y[t], a[0]) and torch.equal(z[t], a[1]) and torch.equal(stats[t], a[2])
    assert torch.equal(grads[0][t], b[0]) and torch.equal(grads[1][t], b[1])
    del grads, y, z, b
    # a sum over all rows: db_pre is dz's (x's), 264 rows a workgroup and 1,024 of those
    got = gt.block_norm_bwd(x, f, stats, f, x, **kw)[6].double()
    ref, size = torch.zeros(D, dtype=torch.float64, device="cuda"), torch.zeros(D, dtype=torch.float64, device="cuda")
    for s in range(0, n, 10_000):
        ref += x[s:s + 10_000].double().sum(0)
        size += x[s:s + 10_000].double().abs().sum(0)
    assert ((got - ref).abs() <= (264 + 16 + 64) * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv", [(256, 256), (256, 16), (10, 5), (24, 12), (7, 7), (112, 7)])
@pytest.mark.parametrize("B", [0, 64])
def test_head_counts(gt, dtype, H, Hkv, B):
    compare(gt, [3, 20, 1], [5, 20, 30], H, Hkv, 32, dtype, True, B, seed=H)
    compare(gt, [40, 2], [70, 33], H, Hkv, 32, dtype, False, B, seed=H + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [0, 64])
@pytest.mark.parametrize("d", [32, 128])
def test_captured_lists_of_every_size_replay(gt, dtype, B, d):
    # single tokens, split walks with their merges, tiles and small sequences; the largest tables
    lq, lk, H = [1, 150, 30, 2, 70], [5000, 150, 30, 3000, 1300], 4
    q, k, v, do, table, ids = make(lq, lk, H, 2, d, dtype, B)
    plan = gt.packed_plan(ptrs(lq), ptrs(lk), heads=H, kv_heads=2, causal=True)
    assert plan.c.layout[28] > 0
    Q, K, V, dO = (dev_feat(x, dtype) for x in (q, k, v, do))
    if B:
        T, I = torch.from_numpy(table).cuda(), torch.from_numpy(ids).cuda()

    def step():
        if B:
            O, L = gt.packed_attn_fwd_bias(plan, Q, K, V, T, I)
            return (O, L) + gt.packed_attn_bwd_bias(plan, Q, K, V, T, I, dO, L)
        O, L = gt.packed_attn_fwd(plan, Q, K, V)
        return (O, L) + gt.packed_attn_bwd(plan, Q, K, V, O, dO, L)

    step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(step())
    for turn in range(3):
        Q.copy_(dev_feat(normal_tensor(q.shape, (turn, 1), dtype), dtype))
        for graph in graphs:
            graph.replay()
        got = [[x.clone() for x in out] for out in outs]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for out in got for x, y in zip(out, want)), turn


@pytest.mark.parametrize("H", [1, 8])
def test_captured_edge_bias_replays(gt, H):
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, 66, (70_003,), dtype=torch.uint8, device="cuda", generator=g)
    table, grad = torch.randn(64, H, device="cuda"), torch.randn(70_003, H, device="cuda")

    def step():
        return gt.bucket_bias_fwd(table, ids), gt.bucket_bias_bwd(ids, grad, 64)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for turn in range(4):
        table.normal_()
        grad.normal_()
        graph.replay()
        got = [x.clone() for x in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), turn
