"""CPU pins of the oracle of embedding, dropout and the class loss: known words of the generator, gradients against
differences, and that the bounds let an fp32 run of the formulas pass and wrong ones not."""

import numpy as np
import pytest
import torch

from oracle import ends as OE

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def inside(x, rb):
    r, b = rb
    return bool(((x.double() - r).abs() <= b).all())


def loss_inputs(n, V, D, dtype, seed=0, labelled=0.8):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, D, generator=g).to(DT[dtype])
    w = (torch.randn(V, D, generator=g) * 2 / D ** 0.5).to(DT[dtype])
    y = torch.randint(0, V, (n,), generator=g)
    y[torch.rand(n, generator=g) > labelled] = -100
    return x, w, y, torch.randn(n, generator=g)


def test_generator_known_words():
    # Philox4x32-10's published answers: zeros; all ones (the counter's high words are zero here, so that one is not
    # reachable); 64-bit counters wrap
    assert [hex(v) for v in OE.philox(0, 0, 1)[0]] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    a = OE.philox(12345678901234567890, 2 ** 64 - 1, 3)
    assert np.array_equal(a[1], OE.philox(12345678901234567890, 0, 1)[0])
    assert np.array_equal(OE.philox(7, 2 ** 32 - 1, 2)[1], OE.philox(7, 2 ** 32, 1)[0])


def test_generator_share_and_independence():
    keep = OE.dropout_keep(400_000, 0.3, 99, 5)
    assert abs(keep.mean() - 0.7) < 5 * np.sqrt(0.21 / 400_000)
    other = OE.dropout_keep(400_000, 0.3, 100, 5)
    assert abs((keep & other).mean() - 0.49) < 0.005
    assert abs((keep[1:] & keep[:-1]).mean() - 0.49) < 0.005
    assert OE.dropout_keep(1000, 0.0, 3, 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_bounds_hold_fp32_and_not_less(dtype):
    half = HALF[dtype]
    for n, V, D in ((5, 3, 8), (40, 130, 64), (70, 33, 100)):
        x, w, y, up = loss_inputs(n, V, D, dtype, seed=n)
        ref = OE.class_loss(x, w, y, up, half)
        has = y >= 0
        rows = torch.where(has, y, 0)
        s = x.float() @ w.float().t()
        lse = torch.logsumexp(s, 1)
        g = torch.exp(s - lse[:, None])
        g[torch.arange(n), rows] -= 1
        g = (g * torch.where(has, up, 0.0)[:, None]).to(DT[dtype]).float()
        loss = torch.where(has, lse - s[torch.arange(n), rows], 0.0)
        good = dict(loss=loss, lse=torch.where(has, lse, 0.0), dx=(g @ w.float()).to(DT[dtype]),
                    dw=(g.t() @ x.float()).to(DT[dtype]))
        for k, v in good.items():
            assert inside(v, ref[k]), (k, n, V, D)
        # a class left out of the sum, a gradient without the label's term or without a class, a dropped row
        bad = lse + torch.log1p(-torch.exp(s[:, -1] - lse))
        assert not inside(torch.where(has, bad, 0.0), ref["lse"])
        h = g.clone()
        h[:, V // 2] = 0
        assert not inside(h @ w.float(), ref["dx"]) and not inside(h.t() @ x.float(), ref["dw"])
        h = g.clone()
        h[int(torch.nonzero(has)[0])] = 0
        assert not inside(h @ w.float(), ref["dx"]) and not inside(h.t() @ x.float(), ref["dw"])


def test_loss_gradient_against_differences():
    x, w, y, up = loss_inputs(6, 7, 5, "f32", seed=3)
    ref = OE.class_loss(x, w, y, up, HALF["f32"])
    x, w = x.double(), w.double()
    total = lambda a, b: (OE.class_loss(a, b, y, up, 0.0)["loss"][0] * up.double()).sum()  # noqa: E731
    for name, base, k in (("dx", x, 0), ("dw", w, 1)):
        for i in range(0, base.numel(), 3):
            d = torch.zeros_like(base).view(-1)
            d[i] = 1e-5
            d = d.view_as(base)
            up_, dn = ((x + d, w) if k == 0 else (x, w + d)), ((x - d, w) if k == 0 else (x, w - d))
            diff = (total(*up_) - total(*dn)) / 2e-5
            assert abs(diff - ref[name][0].view(-1)[i]) < 1e-8


def test_embed_pins():
    table = torch.arange(12.0).view(4, 3)
    ids = torch.tensor([[0, 3], [-1, 1], [4, 4], [3, 3]])
    out, _ = OE.embed(table, ids, 2.0, 0.0)
    assert torch.equal(out, torch.tensor([[18., 22, 26], [6, 8, 10], [0, 0, 0], [36, 40, 44]], dtype=torch.float64))
    grad, b = OE.embed_grad(ids, torch.ones(4, 3), 4, 2.0, 2.0 ** -24)
    assert torch.equal(grad[:, 0], torch.tensor([2., 2, 0, 6], dtype=torch.float64))
    assert (b < 1e-4).all()  # another term would be outside


def test_dropout_bound():
    x, add = torch.randn(1000), torch.randn(1000)
    keep = torch.from_numpy(OE.dropout_keep(1000, 0.25, 1, 2))
    y = torch.where(keep, x * np.float32(1 / 0.75), torch.zeros(())) + add
    assert inside(y, OE.dropout(x, add, keep, 0.25, 2.0 ** -24))
    assert not inside(torch.where(keep, x, torch.zeros(())) + add, OE.dropout(x, add, keep, 0.25, 2.0 ** -24))
