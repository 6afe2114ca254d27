"""GPU embedding, dropout and class loss vs the fp64 oracle, each result held to the bound that the oracle derives for
fp32 arithmetic and one rounding, and to exact results on whole numbers; and the operators together as a model's ends."""

import math
import sys

import numpy as np
import pytest
import torch

from oracle import ends as OE

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
IT = {"i32": torch.int32, "i64": torch.int64}


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def check(name, x, rb):
    r, b = (v.to(x.device) for v in rb)
    assert x.shape == r.shape and bool(torch.isfinite(x).all()), name
    err = (x.double() - r).abs()
    over = err - b
    assert over.numel() == 0 or over.max() <= 0, (f"{name}: {int((over > 0).sum())}/{over.numel()} outside their bound, "
                                                  f"by up to {over.max():.3e} (largest error {err.max():.3e})")


def normal(shape, seed, dtype, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(DT[dtype])


# ---------------------------------------------------------------------------------------------- embedding

def skewed_ids(n, F, R, seed, itype, bad=0.05):
    g = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand(n, F, generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(R + 1.0)) - 1).long().clamp_(0, R - 1)
    ids[torch.rand(n, F, generator=g, device="cuda") < bad] = -1
    ids[torch.rand(n, F, generator=g, device="cuda") < bad / 2] = R
    return ids.to(IT[itype])


def embed_case(gt, n, F, R, D, dtype, itype, scale=1.0, ids=None, seed=0, backward=True):
    say("embed", n, F, R, D, dtype, itype)
    table, dout = normal((R, D), seed + 1, dtype), normal((n, D), seed + 2, dtype)
    ids = skewed_ids(n, F, R, seed + 3, itype) if ids is None else ids
    out = gt.embed_fwd(table, ids, scale)
    torch.cuda.synchronize()
    s = float(np.float32(scale))
    check("out", out, OE.embed(table, ids, s, HALF[dtype]))
    if not backward:
        return out
    grad = gt.embed_bwd(ids, dout, R, scale)
    check("dtable", grad, OE.embed_grad(ids, dout, R, s, HALF[dtype]))
    assert torch.equal(grad, gt.embed_bwd(ids, dout, R, scale))
    return out, grad


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("itype", ["i32", "i64"])
@pytest.mark.parametrize("n,F,R,D", [(1, 1, 1, 1), (1, 1, 5, 3), (3, 2, 7, 7), (7, 1, 100, 8), (16, 1, 1000, 2048),
                                     (65, 3, 11, 9), (64, 1, 2, 64), (300, 9, 173, 100), (1000, 1, 3, 33),
                                     (1025, 5, 4000, 257), (5000, 2, 60_000, 16), (129, 12, 300, 4100), (2000, 1, 1, 511)])
def test_embed(gt, n, F, R, D, dtype, itype):
    embed_case(gt, n, F, R, D, dtype, itype, scale=1.0 if F > 1 else math.sqrt(D), seed=n + D)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_embed_long_runs(gt, dtype):
    # every pair one id; runs of exactly, one less and one more than what a group adds alone, at every place of a chunk
    for n in (63, 64, 65, 127, 128, 129, 4096, 20_001):
        embed_case(gt, n, 1, 9, 72, dtype, "i64", ids=torch.full((n,), 4, dtype=torch.int64, device="cuda"))
    lens = [1, 64, 65, 63, 66, 200, 2, 64, 64, 129, 1, 700, 65]
    ids = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor(lens, device="cuda"))
    perm = torch.randperm(ids.numel(), generator=torch.Generator().manual_seed(1)).cuda()
    embed_case(gt, ids.numel(), 1, len(lens) + 2, 40, dtype, "i32", ids=ids[perm].int())
    embed_case(gt, 30_000, 3, 20, 256, dtype, "i32", seed=4)


def test_embed_whole_numbers(gt):
    # sums of small whole numbers are exact in fp32 in any order: every term is there once, and none twice
    for n, F, R, D in ((50_000, 2, 37, 24), (3000, 1, 5000, 136), (200_000, 1, 3, 8)):
        ids = skewed_ids(n, F, R, n, "i64")
        g = torch.Generator(device="cuda").manual_seed(n)
        dout = torch.randint(-8, 9, (n, D), generator=g, device="cuda").float()
        got = gt.embed_bwd(ids, dout, R)
        want = torch.zeros(R + 1, D, dtype=torch.float64, device="cuda")
        for f in range(F):
            want.index_add_(0, torch.where((ids[:, f] >= 0) & (ids[:, f] < R), ids[:, f], R), dout.double())
        assert torch.equal(got.double(), want[:-1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_embed_tables_of_few_rows(gt, dtype):
    # rows held in LDS: 16 or 8 pieces of 16 bytes, whole ones and a last one that ends with the row; and the limits
    D16, D8 = (256, 150) if dtype == "bf16" else (128, 77)
    for n, F, R, D in ((35_000, 9, 173, D16), (70_000, 8, 256, D8), (70_000, 4, 257, D16), (100_000, 5, 512, D8 + 3),
                       (70_000, 5, 513, D16), (150_000, 4, 1, 129), (10_001, 12, 31, 1000), (3000, 12, 31, 1000)):
        embed_case(gt, n, F, R, D, dtype, "i64" if n % 2 else "i32", seed=n + R, backward=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_embed_shared_rows_taken_together(gt, dtype):
    # more rows than the L2 caches hold, several fields each: the chunks go by the rows they read
    D = 256 if dtype == "bf16" else 128
    embed_case(gt, 70_000, 3, 900, D, dtype, "i32", seed=1)
    embed_case(gt, 70_000, 2, 100_000, D + 1, dtype, "i64", seed=2)


@pytest.mark.parametrize("pairs", [8191, 8192, 8193])
def test_embed_sorts_at_their_limits(gt, pairs):
    # one workgroup's sort and the device-wide one, keys of one to four digits
    for R in (200, 255, 256, 40_000, 70_000, 20_000_000):
        embed_case(gt, pairs, 1, R, 3, "f32", "i64", seed=R % 1000)


# ids of 9, 10, 19, 20 and 29 bits: one to four passes of the sort over the grid, into either array at its end
@pytest.mark.parametrize("R,D", [(511, 40), (512, 40), (300_000, 24), (1 << 20, 8), ((1 << 28) + 3, 1)])
def test_embed_sorts_of_every_number_of_passes(gt, R, D):
    embed_case(gt, 9001, 2, R, D, "bf16", "i64" if R % 2 else "i32", seed=R % 1000)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_embed_widest_rows_and_many_fields(gt, dtype):
    embed_case(gt, 150, 1, 20, gt.GT_MAX_WIDTH, dtype, "i32", seed=1)
    embed_case(gt, 40, 2, 3, gt.GT_MAX_WIDTH - 1, dtype, "i64", seed=2)
    embed_case(gt, 300, 100, 50, 36, dtype, "i32", seed=3)
    embed_case(gt, 2, 5000, 9, 20, dtype, "i64", seed=4)


def test_embed_same_id_in_two_fields(gt):
    ids = torch.randint(0, 7, (300, 1), generator=torch.Generator().manual_seed(0)).cuda().repeat(1, 3).contiguous()
    embed_case(gt, 300, 3, 7, 40, "bf16", "i64", ids=ids)


def test_embed_results_beyond_the_caches(gt):
    embed_case(gt, 150_000, 1, 140_000, 1024, "bf16", "i64", seed=3)
    embed_case(gt, 80_000, 2, 90_000, 1001, "f32", "i32", seed=4)


def test_embed_nothing_and_far_ids(gt):
    table = normal((10, 16), 0, "f32")
    none = torch.empty((0, 3), dtype=torch.int32, device="cuda")
    assert gt.embed_fwd(table, none).shape == (0, 16)
    assert not gt.embed_bwd(none, torch.empty((0, 16), device="cuda"), 10).any()
    far = torch.tensor([-1, 10, -2 ** 62, 2 ** 62, 2 ** 32, -2 ** 31, 2 ** 32 + 3], device="cuda")
    assert not gt.embed_fwd(table, far).any()
    dout = torch.full((far.numel(), 16), float("nan"), device="cuda")
    assert not gt.embed_bwd(far, dout, 10).any()  # what no id names is read by nothing


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_embed_views_off_their_alignment(gt, dtype):
    n, R, D = 200, 50, 100
    for off in (1, 3):
        base = normal((R * D + 8,), 5, dtype)
        table = base[off:off + R * D].view(R, D)
        dout = normal((n * D + 8,), 6, dtype)[off:off + n * D].view(n, D)
        ids = skewed_ids(n, 1, R, 7, "i64")
        check("out", gt.embed_fwd(table, ids), OE.embed(table, ids, 1.0, HALF[dtype]))
        check("dtable", gt.embed_bwd(ids, dout, R), OE.embed_grad(ids, dout, R, 1.0, HALF[dtype]))


# ------------------------------------------------------------------------------------------------ dropout

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.97])
def test_dropout(gt, dtype, p):
    for n in (1, 2, 3, 4, 5, 7, 8, 9, 15, 17, 1023, 4096, 70_001):
        say("dropout", n, dtype, p)
        x, add = normal((n,), n, dtype), normal((n,), n + 1, dtype)
        key, counter = 0x9E3779B97F4A7C15 ^ n, 2 ** 63 - 2 + n
        rng = torch.tensor(np.array([key, counter], dtype=np.uint64).view(np.int64), device="cuda")
        keep = torch.from_numpy(OE.dropout_keep(n, p, key, counter)).cuda()
        y, z = gt.dropout(x, p, rng), gt.dropout(x, p, rng, add=add)
        torch.cuda.synchronize()
        check("y", y, OE.dropout(x, None, keep, p, HALF[dtype]))
        check("y + add", z, OE.dropout(x, add, keep, p, HALF[dtype]))
        assert torch.equal(y != 0, keep & (x != 0))


def test_dropout_drops_what_is_not_a_number(gt):
    n = 5000
    x = torch.full((n,), float("nan"), device="cuda")
    x[::2] = float("inf")
    rng = torch.tensor([3, 4], device="cuda")
    keep = torch.from_numpy(OE.dropout_keep(n, 0.5, 3, 4)).cuda()
    y = gt.dropout(x, 0.5, rng)
    assert not y[~keep].any() and not torch.isfinite(y[keep]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropout_shapes_views_counters(gt, dtype):
    base = normal((1000 + 3,), 1, dtype)
    rng = torch.tensor([-5, -1], device="cuda")  # the counter wraps after the first four elements
    keep = torch.from_numpy(OE.dropout_keep(1000, 0.3, -5, -1)).cuda()
    for off in (0, 1, 3):
        x = base[off:off + 1000].view(10, 100)
        check("y", gt.dropout(x, 0.3, rng), OE.dropout(x, None, keep.view(10, 100), 0.3, HALF[dtype]))
    assert gt.dropout(base[:0], 0.3, rng).numel() == 0
    # a call that starts where another's counters end continues its numbers
    x = normal((64,), 2, dtype)
    whole = gt.dropout(x, 0.5, torch.tensor([9, 100], device="cuda"))
    parts = torch.cat([gt.dropout(x[:32], 0.5, torch.tensor([9, 100], device="cuda")),
                       gt.dropout(x[32:], 0.5, torch.tensor([9, 108], device="cuda"))])
    assert torch.equal(whole, parts)


def test_dropout_in_place(gt):
    lib = gt.load_library()
    for which in (0, 1):
        x, add = normal((4097,), 1, "bf16"), normal((4097,), 2, "bf16")
        rng = torch.tensor([1, 2], device="cuda")
        want = gt.dropout(x, 0.2, rng, add=add)
        y = (x, add)[which]
        assert lib.gt_dropout(4097, gt.GT_BF16, 0.2, rng.data_ptr(), x.data_ptr(), add.data_ptr(), y.data_ptr(),
                              torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert torch.equal(y, want)


# --------------------------------------------------------------------------------------------------- loss

def loss_inputs(n, V, D, dtype, itype, labelled, seed, std=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, w = normal((n, D), seed + 1, dtype), normal((V, D), seed + 2, dtype, std / math.sqrt(D))
    y = torch.randint(0, V, (n,), generator=g, device="cuda")
    off = torch.rand(n, generator=g, device="cuda") >= labelled
    y[off] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, -100, V)[off]
    return x, w, y.to(IT[itype]), torch.randn(n, generator=g, device="cuda")


def loss_case(gt, n, V, D, dtype, itype="i64", labelled=0.8, seed=0, inputs=None, std=2.0):
    say("loss", n, V, D, dtype, itype, labelled)
    x, w, y, up = loss_inputs(n, V, D, dtype, itype, labelled, seed, std) if inputs is None else inputs
    loss, lse = gt.class_loss_fwd(x, w, y)
    dx, dw = gt.class_loss_bwd(x, w, y, lse, up)
    torch.cuda.synchronize()
    ref = OE.class_loss(x, w, y, up, HALF[dtype])
    for name, v in dict(loss=loss, lse=lse, dx=dx, dw=dw).items():
        check(name, v, ref[name])
        if V >= 40 and n >= 20 and std <= 2.0:
            # and as a whole: two roundings of half a step where no sum is smaller than its terms' sizes together; fp32
            # as everywhere
            r = ref[name][0]
            assert (v.double() - r).norm() <= (2.0 ** -7 if dtype == "bf16" else 1e-5) * r.norm(), name
    off = (y < 0) | (y >= V)
    assert not loss[off].any() and not lse[off].any() and not dx[off].any()
    return loss, lse, dx, dw


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,D", [(1, 1, 1), (1, 2, 8), (2, 3, 5), (3, 40, 64), (33, 40, 64), (64, 64, 64), (65, 65, 72),
                                   (7, 2000, 32), (100, 257, 100), (257, 256, 128), (300, 1000, 96), (513, 300, 64),
                                   (64, 513, 256), (1000, 172, 256), (20, 5000, 192), (2500, 47, 33), (130, 700, 1000)])
def test_loss(gt, n, V, D, dtype):
    loss_case(gt, n, V, D, dtype, itype="i32" if n % 2 else "i64", labelled=1.0 if n < 4 else 0.7, seed=n + V + D)


# every shape of block that the logits, dX and dW are formed in at middle sizes, whole and in split sums, with rows
# without a label: the device has fewer rows than the shapes were chosen for
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,D", [(300, 3000, 1100), (1100, 3000, 1100), (2100, 1500, 130), (2100, 3000, 130),
                                   (5000, 6000, 70), (9000, 300, 1100), (9000, 6000, 70), (9000, 1500, 130),
                                   (20_000, 70, 600), (20_000, 300, 600), (20_000, 700, 300), (20_000, 3000, 70)])
def test_loss_in_blocks_of_every_shape(gt, n, V, D, dtype):
    loss_case(gt, n, V, D, dtype, labelled=0.7, seed=n + V + D)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_widest_rows(gt, dtype):
    loss_case(gt, 70, 130, gt.GT_MAX_WIDTH, dtype, seed=1)
    loss_case(gt, 300, 20, gt.GT_MAX_WIDTH - 1, dtype, labelled=0.5, seed=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_one_side_at_a_time(gt, dtype):
    x, w, y, up = loss_inputs(300, 500, 128, dtype, "i64", 0.6, 3)
    lse = gt.class_loss_fwd(x, w, y)[1]
    dx, dw = gt.class_loss_bwd(x, w, y, lse, up)
    only_x, none = gt.class_loss_bwd(x, w, y, lse, up, want_dw=False)
    assert none is None and torch.equal(only_x, dx)
    none, only_w = gt.class_loss_bwd(x, w, y, lse, up, want_dx=False)
    assert none is None and torch.equal(only_w, dw)
    again = gt.class_loss_bwd(x, w, y, lse, up)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_labels_that_leave_nothing(gt, dtype):
    x, w, y, up = loss_inputs(400, 300, 64, dtype, "i64", 1.0, 5)
    for keep in ([], [399], [0, 256], list(range(255, 258))):
        z = torch.full_like(y, -100)
        z[keep] = y[keep]
        loss, lse, dx, dw = loss_case(gt, 400, 300, 64, dtype, inputs=(x, w, z, up))
        if not keep:
            assert not dw.any()
    for far in (2 ** 40, -2 ** 40, 2 ** 32 + 5, 300):
        loss, lse = gt.class_loss_fwd(x, w, torch.full_like(y, far))
        assert not loss.any() and not lse.any()
    e = torch.empty((0, 64), dtype=DT[dtype], device="cuda")
    none = torch.empty(0, device="cuda")
    loss, lse = gt.class_loss_fwd(e, w, y[:0])
    dx, dw = gt.class_loss_bwd(e, w, y[:0], none, none)
    assert loss.numel() == lse.numel() == dx.numel() == 0 and not dw.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [60, 256, 257, 500])
def test_loss_rows_without_a_label_are_not_read_into_results(gt, n, dtype):
    x, w, y, up = loss_inputs(n, 200, 64, dtype, "i64", 0.5, 6)
    off = (y < 0) | (y >= 200)
    want = gt.class_loss_fwd(x, w, y)
    grad = gt.class_loss_bwd(x, w, y, want[1], up)
    x, up = x.clone(), up.clone()
    x[off], up[off] = float("nan"), float("inf")
    got = gt.class_loss_fwd(x, w, y)
    for a, b in zip(want + grad, got + gt.class_loss_bwd(x, w, y, got[1], up)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_strides(gt, dtype):
    for n, V, D, px, pw in ((100, 130, 64, 64, 16), (100, 130, 64, 3, 5), (70, 90, 50, 14, 0), (33, 40, 128, 0, 1)):
        x, w, y, up = loss_inputs(n, V, D, dtype, "i64", 0.9, 8)
        wide_x = torch.full((n, D + px), float("nan"), dtype=DT[dtype], device="cuda")
        wide_w = torch.full((V, D + pw), float("nan"), dtype=DT[dtype], device="cuda")
        wide_x[:, :D], wide_w[:, :D] = x, w
        loss_case(gt, n, V, D, dtype, inputs=(wide_x[:, :D], wide_w[:, :D], y, up))
    x, w, y, up = loss_inputs(9, 20, 64, dtype, "i64", 1.0, 9)
    off = torch.empty(9 * 64 + 1, dtype=DT[dtype], device="cuda")[1:].view(9, 64)
    with pytest.raises(gt.GtError, match="16 bytes"):
        gt.class_loss_fwd(off, w, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_large_logits(gt, dtype):
    # logits of thousands, either sign: nothing overflows, and the loss of a row far from its label is the distance
    x, w, y, up = loss_inputs(70, 300, 64, dtype, "i64", 1.0, 10, std=300.0)
    loss, lse, _, _ = loss_case(gt, 70, 300, 64, dtype, inputs=(x, w, y, up), std=300.0)  # exp of numbers 1e-3 off
    assert loss.max() > 1000
    same = torch.zeros_like(w)
    loss, lse = gt.class_loss_fwd(x, same, y)
    assert (lse - math.log(300)).abs().max() < 1e-5 and (loss - math.log(300)).abs().max() < 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_pieces_and_split_sums(gt, dtype):
    # many rows and more classes than a piece holds; few rows and a long sum for dX; few classes and a long one for dW
    for n, V, D, lab in ((70_000, 3000, 64, 0.9), (100, 40_000, 64, 1.0), (60_000, 30, 64, 0.5), (9000, 300, 128, 0.1)):
        loss_case(gt, n, V, D, dtype, labelled=lab, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_equal_upstream_gradients_are_exact_factors(gt, dtype):
    # a mean: what is rounded to bf16 does not depend on 1 / m, so another m scales every gradient by the ratio alone
    x, w, y, _ = loss_inputs(300, 500, 64, dtype, "i64", 0.7, 11)
    lse = gt.class_loss_fwd(x, w, y)[1]
    a = gt.class_loss_bwd(x, w, y, lse, torch.full((300,), 1.0, device="cuda"))
    b = gt.class_loss_bwd(x, w, y, lse, torch.full((300,), 1.0 / 6963, device="cuda"))
    for p, q in zip(a, b):
        # two roundings to the features' type, and a few of fp32
        assert ((p.double() / 6963 - q.double()).abs() <= (2 * HALF[dtype] + 8 * 2.0 ** -24) * q.double().abs()).all()
    zero = gt.class_loss_bwd(x, w, y, lse, torch.zeros(300, device="cuda"))
    assert not zero[0].any() and not zero[1].any()
    tiny = torch.full((300,), 1e-36, device="cuda")
    big = torch.full((300,), 1e30, device="cuda")
    for up in (tiny, big):
        for p, q in zip(a, gt.class_loss_bwd(x, w, y, lse, up)):
            f = float(up[0])
            # fp32 has no finer numbers than 2^-149, and bf16 none below 2^-133
            assert ((p.double() * f - q.double()).abs() <= (2 * HALF[dtype] + 2.0 ** -20) * q.double().abs() + 2.0 ** -132).all()


@pytest.mark.parametrize("n", [255, 256, 257, 8192, 8193])
def test_loss_listed_rows_at_their_limits(gt, n):
    loss_case(gt, n, 70, 64, "bf16", labelled=0.5, seed=n)
    loss_case(gt, n, 2049, 32, "f32", labelled=0.9, seed=n)  # X's rows laid out once


# ----------------------------------------------------------------------------- streams, graphs, together

def test_other_stream_and_captured_replays(gt):
    """The three operators of a step captured into a graph: replays on new inputs, with eager work between them, give
    what the eager calls give; the generator's numbers come from the device at replay."""
    n, R, D, V = 700, 300, 128, 400
    ids = skewed_ids(n, 2, R, 1, "i64")
    table, w = normal((R, D), 2, "bf16"), normal((V, D), 3, "bf16", 0.1)
    labels = torch.randint(0, V, (n,), device="cuda")
    labels[::5] = -1
    rng, up = torch.tensor([5, 0], device="cuda"), torch.full((n,), 1.0 / n, device="cuda")

    def step():
        x = gt.embed_fwd(table, ids, 2.0)
        h = gt.dropout(x, 0.2, rng, add=x)
        loss, lse = gt.class_loss_fwd(h, w, labels)
        dh, dw = gt.class_loss_bwd(h, w, labels, lse, up)
        dx = gt.dropout(dh, 0.2, rng, add=dh)
        return x, h, loss, lse, dh, dw, dx, gt.embed_bwd(ids, dx, R, 2.0)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = step()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, step()):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(4):
        ids.copy_(skewed_ids(n, 2, R, 10 + k, "i64"))
        labels.copy_(torch.randint(-3, V, (n,), device="cuda"))
        rng[1] += 1000
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in got]
        for a, b in zip(kept, step()):
            assert torch.equal(a, b), k


def test_two_captured_steps_that_share_memory(gt):
    """Two graphs of one pool, replayed in turn with eager work between them, at sizes where every kernel of a large call
    runs: the sort over the grid, long runs, rows taken together, listed and laid-out rows, joined statistics."""
    cases = []
    for k, (n, R, D, V) in enumerate([(20_000, 1000, 1024, 3000), (30_000, 700, 640, 300)]):
        ids, w = skewed_ids(n, 2, R, k, "i32"), normal((V, D), 10 + k, "bf16", 0.05)
        labels = torch.randint(-V // 4, V, (n,), device="cuda")
        x, up = normal((n, D), 20 + k, "bf16"), torch.full((n,), 1.0 / n, device="cuda")
        cases.append((x, w, labels, up, ids, torch.tensor([k, 3], device="cuda"), R))

    def step(x, w, labels, up, ids, rng, R):
        h = gt.dropout(x, 0.3, rng)
        loss, lse = gt.class_loss_fwd(h, w, labels)
        dh, dw = gt.class_loss_bwd(h, w, labels, lse, up)
        return loss, lse, dh, dw, gt.embed_bwd(ids, dh, R)

    for c in cases:
        step(*c)
    torch.cuda.synchronize()
    graphs, got = [], []
    for c in cases:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], pool=graphs[0].pool() if len(graphs) > 1 else None):
            got.append(step(*c))
    for k in (0, 1, 1, 0, 1, 0):
        c = cases[k]
        c[0].copy_(normal(c[0].shape, 100 + k, "bf16"))
        c[2].copy_(c[2].roll(17))
        c[5][1] += 10_000_000
        graphs[k].replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in got[k]]
        for a, b in zip(kept, step(*c)):
            assert torch.equal(a, b), k


def test_a_model_from_ids_to_loss(gt):
    """Embedding, dropout, packed attention, the norms between blocks and the loss, with the table as the classes'
    weights: the gradients of the table follow those of the same model in 64 bits."""
    lens, R, H, d = [40, 7, 100, 1, 64], 90, 4, 32
    n, D, p = sum(lens), H * d, 0.25
    ptr = torch.tensor([0] + list(np.cumsum(lens)))
    plan = gt.packed_plan(ptr, heads=H, causal=True)
    table = normal((R, D), 1, "f32", 0.3)
    ids = skewed_ids(n, 1, R, 2, "i64", bad=0.0)[:, 0].contiguous()
    labels = torch.where(torch.arange(n, device="cuda") % 4 == 0, -1, (ids * 7 + 3) % R)
    rng = torch.tensor([11, 50], device="cuda")
    up = torch.full((n,), 1.0, device="cuda") / (labels >= 0).sum()
    x = gt.embed_fwd(table, ids, 2.0)
    q = x.view(n, H, d)
    o, lse_a = gt.packed_attn_fwd(plan, q, q, q)
    f = gt.dropout(o.view(n, D), p, rng)
    y, z, stats = gt.block_norm_fwd(x, f, kind="rms")
    loss, lse = gt.class_loss_fwd(z, table, labels)
    dz, dw = gt.class_loss_bwd(z, table, labels, lse, up)
    dx, df, *_ = gt.block_norm_bwd(x, f, stats, torch.zeros_like(y), dz, kind="rms")
    do = gt.dropout(df, p, rng).view(n, H, d)
    dq, dk, dv = gt.packed_attn_bwd(plan, q, q, q, o, do, lse_a)
    grad = gt.embed_bwd(ids, dx + (dq + dk + dv).view(n, D), R, 2.0) + dw

    t = table.double().requires_grad_()
    X = t[ids] * 2.0
    keep = torch.from_numpy(OE.dropout_keep(n * D, p, 11, 50)).cuda().view(n, D)
    rows = []
    for a, b in zip(ptr[:-1].tolist(), ptr[1:].tolist()):
        Q = X[a:b].view(b - a, H, d).transpose(0, 1)
        s = Q @ Q.transpose(1, 2) / math.sqrt(d)
        s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        rows.append((torch.softmax(s, -1) @ Q).transpose(0, 1).reshape(b - a, D))
    F = torch.where(keep, torch.cat(rows) / (1 - p), 0.0)
    unit = lambda v: v * torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-5)  # noqa: E731
    Z = unit(X + unit(F))
    has = labels >= 0
    logits = Z @ t.t()
    L = torch.where(has, torch.logsumexp(logits, 1) - logits.gather(1, labels.clamp(min=0)[:, None])[:, 0], 0.0)
    (want,) = torch.autograd.grad((L * up.double()).sum(), [t])
    # fp32 throughout: about 40 roundings of values of the size of the results' own, most of them independent
    assert (loss.double() - L).abs().max() <= 1e-4 * L.abs().max()
    assert (grad.double() - want).norm() <= 1e-4 * want.norm()
