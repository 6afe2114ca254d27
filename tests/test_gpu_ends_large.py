"""GPU embedding, dropout and class loss where offsets pass 32 bits, over more classes than one launch takes, and from
two streams at once."""

import math

import pytest
import torch

from oracle import ends as OE
from tests.test_gpu_ends import HALF, check, loss_inputs, normal, say, skewed_ids

pytestmark = pytest.mark.gpu

FAR = (1 << 32) // 2048 // 2  # rows of 2,048 bf16 elements that reach 2^32 bytes


def test_embedding_table_and_output_beyond_4_gib(gt):
    n, R, D = 300, FAR + 70_000, 2048
    say("embed far", R, D)
    table = torch.empty((R, D), dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 1, FAR - 1, FAR, FAR + 1, R - 1], device="cuda")
    table[rows] = normal((6, D), 1, "bf16")
    ids = rows[torch.randint(0, 6, (n, 2), generator=torch.Generator().manual_seed(0)).cuda()]
    small = torch.searchsorted(rows, ids)
    check("out", gt.embed_fwd(table, ids), OE.embed(table[rows], small, 1.0, HALF["bf16"]))
    del table
    dout = normal((n, D), 2, "bf16")
    grad = gt.embed_bwd(ids, dout, R)
    check("dtable", grad[rows], OE.embed_grad(small, dout, 6, 1.0, HALF["bf16"]))
    grad[rows] = 0
    assert not grad.view(torch.int16).any()
    del grad
    n = FAR + 5000  # and as many output rows, and rows of dout
    table = normal((50, D), 3, "bf16")
    ids = torch.arange(n, device="cuda").remainder_(53).int()
    out = gt.embed_fwd(table, ids)
    at = torch.tensor([0, 52, FAR - 1, FAR, FAR + 40, n - 1], device="cuda")
    check("far rows", out[at], OE.embed(table, ids[at], 1.0, HALF["bf16"]))
    keep = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    keep[at] = ids[at]
    grad = gt.embed_bwd(keep, out, 50)
    check("far gradients", grad, OE.embed_grad(ids[at], out[at], 50, 1.0, HALF["bf16"]))


def test_dropout_of_more_than_2_to_the_32_elements(gt):
    n = (1 << 32) + 4096 + 5
    say("dropout far", n)
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    rng = torch.tensor([77, 5], device="cuda")
    y = gt.dropout(x, 0.5, rng)
    for start in (0, (1 << 31) - 512, (1 << 32) - 512, n - 4101):
        start -= start % 4
        rng2 = torch.tensor([77, 5 + start // 4], device="cuda")
        m = min(4096, n - start)
        assert torch.equal(y[start:start + m], gt.dropout(x[start:start + m].clone(), 0.5, rng2))


@pytest.mark.parametrize("side", ["rows", "classes"])
def test_loss_beyond_4_gib(gt, side):
    D = 2048
    if side == "rows":  # labelled rows at both ends of 4.5 GB of features
        n, V = FAR + 70_000, 300
        say("loss far rows", n)
        x = torch.empty((n, D), dtype=torch.bfloat16, device="cuda")
        y = torch.full((n,), -1, device="cuda")
        up = torch.empty(n, device="cuda")
        at = torch.cat([torch.arange(60), torch.arange(FAR - 100, FAR + 200), torch.arange(n - 50, n)]).cuda()
        xs, w, ys, ups = loss_inputs(at.numel(), V, D, "bf16", "i64", 1.0, 1)
        x[at], y[at], up[at] = xs, ys, ups
        loss, lse = gt.class_loss_fwd(x, w, y)
        dx, dw = gt.class_loss_bwd(x, w, y, lse, up)
        ref = OE.class_loss(xs, w, ys, ups, HALF["bf16"])
        for name, v in dict(loss=loss[at], lse=lse[at], dx=dx[at], dw=dw).items():
            check(name, v, ref[name])
        dx[at], loss[at] = 0, 0
        assert not dx.view(torch.int16).any() and not loss.any()
        return
    n, V = 40, FAR + 70_000  # 4.5 GB of class weights: most classes are zeros, whose logits are 0
    say("loss far classes", V)
    some = torch.cat([torch.arange(300), torch.arange(FAR - 100, FAR + 200), torch.arange(V - 50, V)]).cuda()
    w = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    xs, ws, ys, up = loss_inputs(n, some.numel(), D, "bf16", "i64", 1.0, 2)
    w[some] = ws
    y = some[ys]
    loss, lse = gt.class_loss_fwd(xs, w, y)
    s = xs.double() @ ws.double().t()
    rest = math.log(V - some.numel())
    want = torch.logsumexp(torch.cat([s, torch.full((n, 1), rest, dtype=torch.float64, device="cuda")], 1), 1)
    # as the oracle bounds them: the logits' 2,048 terms, the sums over the blocks of 256 classes, a few roundings
    ds = D * 2 * OE.U * (xs.double().abs() @ ws.double().abs().t()).amax(1)
    tol = ds + OE.U * (90 + 3 * (V // 256)) + 8 * OE.U * (1 + want.abs() + s.abs().amax(1))
    assert ((lse.double() - want).abs() <= tol).all()
    assert ((loss.double() - (want - s[torch.arange(n), ys])).abs() <= 2 * tol).all()
    dx, dw = gt.class_loss_bwd(xs, w, y, lse, up)
    p = torch.exp(s - want[:, None])
    p[torch.arange(n), ys] -= 1
    p *= up[:, None].double()
    for got, r, size in ((dx, p @ ws.double(), p.abs() @ ws.double().abs()),
                         (dw[some], p.t() @ xs.double(), p.abs().t() @ xs.double().abs())):
        # a rounding of dL, one of the result, and what the logits' and lse's errors make of exp
        assert ((got.double() - r).abs() <= 2.0 ** -8 * r.abs() + (2.0 ** -8 + 3 * float(tol.max())) * size + 1e-30).all()


def test_loss_over_more_classes_than_a_launch_takes(gt):
    # 2^22 blocks a launch: at 200,000 rows, 5,363 blocks of 256 classes, and the forward takes two launches
    n, V, D = 200_000, 5363 * 256 + 700, 64
    say("loss classes", V)
    at = torch.arange(0, n, 4999, device="cuda")
    m = at.numel()
    x, y = torch.empty((n, D), dtype=torch.bfloat16, device="cuda"), torch.full((n,), -1, device="cuda")
    xs, w = normal((m, D), 1, "bf16"), normal((V, D), 2, "bf16", 0.25)
    ys = torch.arange(m, device="cuda") * (V // m)
    ys[:4] = torch.tensor([5363 * 256 - 1, 5363 * 256, V - 1, 0])
    x[at], y[at] = xs, ys
    loss, lse = gt.class_loss_fwd(x, w, y)
    ref = OE.class_loss(xs, w, ys, torch.ones(m, device="cuda"), HALF["bf16"])
    check("loss", loss[at], ref["loss"])
    check("lse", lse[at], ref["lse"])


def test_two_streams_at_once(gt):
    cases = []
    for k in range(2):
        x, w, y, up = loss_inputs(900 + k, 3000, 256, "bf16", "i64", 0.7, 20 + k)
        ids = skewed_ids(9000, 2, 500, 30 + k, "i64")
        cases.append((x, w, y, up, ids, normal((9000, 256), 40 + k, "bf16"), torch.tensor([k, 9], device="cuda")))

    def step(c):
        x, w, y, up, ids, dout, rng = c
        loss, lse = gt.class_loss_fwd(x, w, y)
        return (loss, lse) + gt.class_loss_bwd(x, w, y, lse, up) + (gt.embed_bwd(ids, dout, 500), gt.dropout(dout, 0.3, rng))

    want = [step(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for c, st in zip(cases, streams):
            with torch.cuda.stream(st):
                got.append(step(c))
        torch.cuda.synchronize()
        for g, r in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, r))
