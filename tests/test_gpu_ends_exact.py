"""GPU embedding, dropout and class loss where results can be said exactly or nearly so: the order of an embedding's sums,
products of every number of steps, losses of rows that are sure of their label."""

import pytest
import torch

from oracle import ends as OE
from tests.test_gpu_ends import DT, HALF, check, loss_case, loss_inputs, say

pytestmark = pytest.mark.gpu


def sums_in_order(ids, dout, R, turned=False):
    """fp32 sums of dout's rows for each table row, term after term in the order of the (row, field) pairs."""
    (n, F), d = ids.shape, dout.cpu()
    key = torch.where((ids >= 0) & (ids < R), ids.long(), R).cpu().reshape(-1)
    key, order = torch.sort(key, stable=True)
    first = torch.searchsorted(key, torch.arange(R + 1))
    count, rows = first[1:] - first[:-1], order // F
    out = torch.zeros((R, d.shape[1]))
    for k in range(int(count.max())):
        r = torch.nonzero(count > k)[:, 0]
        out[r] += d[rows[first[r] + (count[r] - 1 - k if turned else k)]]
    return out, int(count.max())


# one workgroup's sort and the grid's, of one to four passes; a width below a piece's and above
@pytest.mark.parametrize("n,F,R,D", [(700, 1, 20, 3), (4000, 2, 300, 20), (8192, 1, 40_000, 8), (8193, 1, 300, 5),
                                     (9000, 3, 900, 20), (20_000, 1, 2000, 36), (30_000, 2, 300_000, 8),
                                     (10_000, 1, 1 << 27, 1)])
def test_embed_terms_are_added_in_order(gt, n, F, R, D):
    # runs of at most 64 terms are one sum, in the order of the tokens: the sort is stable, and no pair is lost or
    # doubled.  Sizes of the terms over ten powers of ten, so that another order rounds otherwise
    say("embed order", n, F, R, D)
    g = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.randint(0, R, (n, F), generator=g, device="cuda")
    ids = torch.where(torch.rand(n, F, generator=g, device="cuda") < 0.03, -1, ids)
    size = 10.0 ** (torch.rand(n, 1, generator=g, device="cuda") * 10 - 5)
    dout = torch.randn(n, D, generator=g, device="cuda") * size
    small = torch.unique(ids[ids >= 0])[:40_000]  # of a large table the rows that are named
    want, most = sums_in_order(torch.searchsorted(small, ids).masked_fill(ids < 0, -1), dout, small.numel())
    assert most <= 64
    if R <= 2000:
        assert not torch.equal(want, sums_in_order(ids, dout, R, turned=True)[0][small.cpu()])
    got = gt.embed_bwd(ids, dout, R)
    assert torch.equal(got[small].cpu(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5])
def test_loss_products_of_every_number_of_steps(gt, dtype, steps):
    # the sum over the features, over the classes and over the rows in one to five steps of 128 bytes: the first step
    # stands alone or in a pair, and its operands have landed in either case
    k = steps * (64 if dtype == "bf16" else 32)
    for n, V, D in ((33, 40, k), (300, 300, k), (1100, 3000, k), (40, k, 96), (k, 70, 64), (250, k, 700)):
        loss_case(gt, n, V, D, dtype, labelled=1.0 if n <= 256 else 0.7, seed=n + V + D)

# one block of classes, a few blocks (joined by a lane a token) and many (by 64 lanes), listed rows and not
SIZES = [(33, 200), (300, 200), (40, 1500), (700, 2000), (50, 5000), (400, 9000)]


def whole_logits(n, V, D, dtype, scale, seed):
    """Features and weights of small whole numbers and multiples of `scale`, a power of two: every logit is exact."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randint(-4, 5, (n, D), generator=g, device="cuda").to(DT[dtype]) * scale
    w = torch.randint(-4, 5, (V, D), generator=g, device="cuda").to(DT[dtype])
    return x, w, x.double() @ w.double().t().contiguous()


def rest_of(s, y):
    """The other classes' sum relative to class y's term, log of it and one, and sum of p |s - s_y|."""
    d = s - s.gather(1, y[:, None])
    other = torch.exp(d).scatter_(1, y[:, None], 0.0)
    p = other / (1 + other.sum(1, keepdim=True))
    return other.sum(1), torch.log1p(other.sum(1)), (p * d.abs()).sum(1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", SIZES)
def test_loss_of_rows_sure_of_their_label(gt, dtype, n, V):
    # the label's logit is the largest: the loss is what the other classes add to the sum, however large the logits are.
    # Its error: the sum's additions (a lane's 64 classes, then the blocks: at most 90 + 3 V / 64), each off by at most
    # half a step of the sum and by no more than what is added; the exponents' (a difference, a rounded constant, a
    # product, exp's own); the logarithm's, a rounded constant and a product
    say("loss sure", n, V, dtype)
    for scale in (1.0 / 32, 0.25, 1.0, 8.0):
        x, w, s = whole_logits(n, V, 64, dtype, scale, n + V)
        y = s.argmax(1)
        loss, lse = gt.class_loss_fwd(x, w, y)
        other, want, size = rest_of(s, y)
        u, adds = 2.0 ** -24, 90 + 3 * (V // 64)
        bound = adds * torch.minimum(u * (1 + other), other) + 4 * u * size + 4 * u * want + 2 * u * want
        assert (loss >= 0).all()
        assert ((loss.double() - want).abs() <= bound).all(), (scale, float((loss.double() - want).abs().max()))
        top = s.amax(1)
        assert ((lse.double() - (top + want)).abs() <= bound + u * (top + want).abs()).all()
        sure = other < 2.0 ** -30  # no sum in fp32 shows the others
        assert scale < 1 or sure.any()
        assert (lse[sure].double() == top[sure]).all() and (loss[sure].double() <= bound[sure]).all()
        # and the label's own gradient is the others' sum, not the rounding of lse
        up = torch.where(sure, 1.0, 0.0)
        dx, dw = gt.class_loss_bwd(x, w, y, lse, up)
        most = 2.0 ** -30 * 4 * max(1.0, 4 * scale) * 2
        assert dx.abs().max() <= most and dw.abs().max() <= n * most
        # at another label it is the distance too
        z = (y + 1) % V
        far = gt.class_loss_fwd(x, w, z)[0].double()
        gap = (top - s.gather(1, z[:, None])[:, 0])
        assert ((far - (gap + want)).abs() <= bound + 2 * u * (gap + want)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 60, 500])
def test_loss_of_one_class_is_nothing(gt, dtype, n):
    for scale in (0.125, 1.0, 16.0):
        x, w, s = whole_logits(n, 1, 100, dtype, scale, n)
        y = torch.zeros(n, dtype=torch.int64, device="cuda")
        loss, lse = gt.class_loss_fwd(x, w, y)
        assert not loss.any() and torch.equal(lse.double(), s[:, 0])
        dx, dw = gt.class_loss_bwd(x, w, y, lse, torch.ones(n, device="cuda"))
        assert not dx.any() and not dw.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", SIZES)
def test_loss_of_near_rows_is_not_negative(gt, dtype, n, V):
    # weights of any value, the features along a class's own
    g = torch.Generator(device="cuda").manual_seed(n)
    w = torch.randn(V, 64, generator=g, device="cuda").to(DT[dtype])
    y = torch.randint(0, V, (n,), generator=g, device="cuda")
    for scale in (0.3, 1.0, 3.0, 15.0):
        x = (w[y].float() * scale).to(DT[dtype])
        s = x.double() @ w.double().t().contiguous()
        at = s.argmax(1)
        loss, lse = gt.class_loss_fwd(x, w, at)
        other, want, _ = rest_of(s, at)
        # two logits' errors (64 terms, in size up to 64 of the label's) move a term of the sum
        ds = 2 * 64 * 2 * 2.0 ** -24 * (x.double().abs() @ w.double().abs().t().contiguous()).amax(1)
        assert (loss >= 0).all()
        assert (loss.double() <= (1.01 + 2 * ds) * want + (90 + 3 * (V // 64)) * torch.minimum(2.0 ** -24 * (1 + other),
                                                                                             other)).all()


# dL of all rows over 1,024 classes, or over all of fewer, beyond 1 GB: the rows too go by in parts, of which the last
# ones may hold no labelled row
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,D,labelled", [(600_000, 1030, 40, 0.9), (560_000, 2100, 24, 1.0), (900_000, 640, 72, 0.2),
                                            (1_100_000, 1000, 256, 0.95), (2_900_000, 200, 24, 0.5)])
def test_loss_rows_in_parts(gt, n, V, D, labelled, dtype):
    x, w, y, up = loss_inputs(n, V, D, dtype, "i64", labelled, n + V)
    loss, lse = gt.class_loss_fwd(x, w, y)
    dx, dw = gt.class_loss_bwd(x, w, y, lse, up)
    say("loss parts", n, V, D, dtype, labelled)
    # the oracle in parts of its own
    at = torch.arange(0, n, 97, device="cuda")
    ref = OE.class_loss(x[at], w, y[at], up[at], HALF[dtype])
    for name, v in dict(loss=loss[at], lse=lse[at], dx=dx[at]).items():
        check(name, v, ref[name])
    r, b = torch.zeros(V, D, dtype=torch.float64, device="cuda"), torch.zeros(V, D, dtype=torch.float64, device="cuda")
    for k in range(0, n, 35_000):
        p, q = OE.class_loss(x[k:k + 35_000], w, y[k:k + 35_000], up[k:k + 35_000], HALF[dtype], rows=n)["dw"]
        r += p
        b += q - HALF[dtype] * p.abs()
    check("dw", dw, (r, b + HALF[dtype] * r.abs()))
    # and as a whole: two roundings of half a step; in fp32 additions to sums that grow as the root of their terms
    assert (dw.double() - r).norm() <= (2.0 ** -7 if dtype == "bf16" else 2.0 ** -24 * (n ** 0.5 + 100)) * r.norm()
    off = (y < 0) | (y >= V)
    assert not loss[off].any() and not lse[off].any() and not dx[off].any()
    only = gt.class_loss_bwd(x, w, y, lse, up, want_dx=False)[1]
    assert torch.equal(only, dw) and torch.equal(gt.class_loss_bwd(x, w, y, lse, up, want_dw=False)[0], dx)


@pytest.mark.parametrize("n,V,D", [(300, 257, 128), (2000, 172, 256), (1500, 5000, 192), (256, 40, 64)])
def test_loss_gradients_in_norm(gt, n, V, D):
    # bf16, upstream gradients over four powers of ten: two roundings, of dL and of the result.  A rounding is off by at
    # most 2^-8 of its value and evenly spread below that: 2^-8 / sqrt 3 in the mean square, two of them 0.82 x 2^-8 where
    # they are independent.  2^-8 leaves room for no third
    x, w, y, up = loss_inputs(n, V, D, "bf16", "i64", 0.8, n + V)
    up = up * 10.0 ** torch.linspace(-4, 0, n)[torch.randperm(n, generator=torch.Generator().manual_seed(n))].cuda()
    lse = gt.class_loss_fwd(x, w, y)[1]
    ref = OE.class_loss(x, w, y, up, HALF["bf16"])
    for name, v in zip(("dx", "dw"), gt.class_loss_bwd(x, w, y, lse, up)):
        check(name, v, ref[name])
        assert (v.double() - ref[name][0]).norm() <= 2.0 ** -8 * ref[name][0].norm(), name
