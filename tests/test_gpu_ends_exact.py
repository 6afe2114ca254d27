"""GPU embedding, dropout and class loss where results can be said exactly or nearly so: the order of an embedding's sums,
products of every number of steps, losses of rows that are sure of their label."""

import pytest
import torch

from tests.test_gpu_ends import loss_case, say

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
