"""Embedding, dropout and the class loss refuse what they do not take, on the host (no GPU)."""

import ctypes
import os

import pytest
import torch

from paper_2407_14106_amd import gt

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced
ODD = ctypes.c_void_p(0x1004)
BIG = 1 << 50
BF, F32, I32, I64 = gt.GT_BF16, gt.GT_F32, gt.GT_I32, gt.GT_I64
ARG, UNS, WS = gt.GT_ERR_INVALID_ARG, gt.GT_ERR_UNSUPPORTED, gt.GT_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gt.LIB_PATH):
        from paper_2407_14106_amd import build

        build.build()
    return gt.load_library()


@pytest.mark.parametrize("n,F,R,D,dt,it,want", [
    (-1, 1, 10, 8, BF, I32, ARG), (1 << 31, 1, 10, 8, BF, I32, ARG), (1 << 30, 2, 10, 8, BF, I32, ARG),
    (5, 0, 10, 8, BF, I32, ARG), (5, -1, 10, 8, BF, I32, ARG), (5, 1, 0, 8, BF, I32, ARG),
    (5, 1, 1 << 31, 8, BF, I32, ARG), (5, 1, 10, 0, BF, I32, ARG), (5, 1, 10, gt.GT_MAX_WIDTH + 1, BF, I32, ARG),
    (5, 1, 10, 8, 2, I32, UNS), (5, 1, 10, 8, F32, 2, UNS)])
def test_embed_sizes(lib, n, F, R, D, dt, it, want):
    assert lib.gt_embed_fwd(n, F, R, D, dt, it, FAKE, FAKE, 1.0, FAKE, None) == want
    assert lib.gt_embed_bwd(n, F, R, D, dt, it, FAKE, FAKE, 1.0, FAKE, FAKE, BIG, None) == want
    if it == I32:
        assert lib.gt_embed_bwd_workspace_size(n, F, R, D, dt) == 0


def test_embed_pointers_and_workspace(lib):
    for args in ((None, FAKE, 1.0, FAKE), (FAKE, None, 1.0, FAKE), (FAKE, FAKE, 1.0, None)):
        assert lib.gt_embed_fwd(5, 1, 10, 8, BF, I64, *args, None) == ARG
    assert lib.gt_embed_fwd(0, 1, 10, 8, BF, I64, None, FAKE, 1.0, None, None) == gt.GT_OK
    need = lib.gt_embed_bwd_workspace_size(500, 2, 10, 8, BF)
    assert need > 0
    for args in ((None, FAKE, 1.0, FAKE, FAKE, BIG), (FAKE, None, 1.0, FAKE, FAKE, BIG),
                 (FAKE, FAKE, 1.0, None, FAKE, BIG), (FAKE, FAKE, 1.0, FAKE, None, BIG)):
        assert lib.gt_embed_bwd(500, 2, 10, 8, BF, I64, *args, None) == ARG
    assert lib.gt_embed_bwd(500, 2, 10, 8, BF, I64, FAKE, FAKE, 1.0, FAKE, FAKE, need - 1, None) == WS


def test_dropout_arguments(lib):
    d = lib.gt_dropout
    assert d(5, 2, 0.1, FAKE, FAKE, None, FAKE, None) == UNS
    assert d(-1, BF, 0.1, FAKE, FAKE, None, FAKE, None) == ARG
    assert d(1 << 48, BF, 0.1, FAKE, FAKE, None, FAKE, None) == ARG
    for p in (-0.1, 1.0, 1.5, float("nan"), float("inf"), 1.0 - 2.0 ** -40):
        assert d(5, BF, p, FAKE, FAKE, None, FAKE, None) == ARG, p
    for args in ((None, FAKE, None, FAKE), (FAKE, None, None, FAKE), (FAKE, FAKE, None, None)):
        assert d(5, BF, 0.1, *args, None) == ARG
    assert d(5, BF, 0.1, ODD, FAKE, None, FAKE, None) == UNS
    assert d(0, BF, 0.1, None, None, None, None, None) == gt.GT_OK


@pytest.mark.parametrize("n,V,D,dt,it,ldx,ldw,want", [
    (-1, 10, 8, BF, I32, 8, 8, ARG), (1 << 28, 10, 8, BF, I32, 8, 8, ARG), (5, 0, 8, BF, I32, 8, 8, ARG),
    (5, 1 << 31, 8, BF, I32, 8, 8, ARG), (5, 10, 0, BF, I32, 8, 8, ARG), (5, 10, 8, BF, I32, 7, 8, ARG),
    (5, 10, 8, BF, I32, 8, 7, ARG), (5, 10, 8, BF, I32, 1 << 31, 8, ARG),
    (5, 10, gt.GT_MAX_WIDTH + 1, BF, I32, 1 << 20, 1 << 20, ARG), (5, 10, 8, 2, I32, 8, 8, UNS),
    (5, 10, 8, F32, 2, 8, 8, UNS)])
def test_loss_sizes(lib, n, V, D, dt, it, ldx, ldw, want):
    assert lib.gt_class_loss_fwd(n, V, D, dt, it, FAKE, ldx, FAKE, ldw, FAKE, FAKE, FAKE, FAKE, BIG, None) == want
    assert lib.gt_class_loss_bwd(n, V, D, dt, it, FAKE, ldx, FAKE, ldw, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, BIG,
                                 None) == want
    if it == I32:
        assert lib.gt_class_loss_fwd_workspace_size(n, V, D, dt, ldx, ldw) == 0
        assert lib.gt_class_loss_bwd_workspace_size(n, V, D, dt, ldx, ldw) == 0


def test_loss_pointers_alignment_workspace(lib):
    fwd = lambda X=FAKE, W=FAKE, y=FAKE, loss=FAKE, lse=FAKE, ws=FAKE, size=BIG, n=50: lib.gt_class_loss_fwd(  # noqa: E731
        n, 10, 64, BF, I64, X, 64, W, 64, y, loss, lse, ws, size, None)
    bwd = lambda X=FAKE, W=FAKE, y=FAKE, lse=FAKE, up=FAKE, dX=FAKE, dW=FAKE, ws=FAKE, size=BIG, n=50: (  # noqa: E731
        lib.gt_class_loss_bwd(n, 10, 64, BF, I64, X, 64, W, 64, y, lse, up, dX, dW, ws, size, None))
    for name in ("X", "W", "y", "loss", "lse", "ws"):
        assert fwd(**{name: None}) == ARG, name
    for name in ("X", "W", "y", "lse", "up", "ws"):
        assert bwd(**{name: None}) == ARG, name
    for name in ("X", "W"):
        assert fwd(**{name: ODD}) == UNS and bwd(**{name: ODD}) == UNS
    need = lib.gt_class_loss_fwd_workspace_size(50, 10, 64, BF, 64, 64)
    assert need > 0 and fwd(size=need - 1) == WS
    need = lib.gt_class_loss_bwd_workspace_size(50, 10, 64, BF, 64, 64)
    assert need > 0 and bwd(size=need - 1) == WS
    assert fwd(n=0, loss=None, lse=None, ws=None) == gt.GT_OK
    assert lib.gt_class_loss_fwd_workspace_size(0, 10, 64, BF, 64, 64) > 0  # no rows, no division by them
    assert lib.gt_class_loss_bwd_workspace_size(0, 10, 64, BF, 64, 64) > 0
    assert lib.gt_embed_bwd_workspace_size(0, 1, 10, 8, BF) > 0
    assert bwd(dX=None, dW=None) == gt.GT_OK  # nothing wanted
    assert bwd(n=0, dW=None) == gt.GT_OK


def test_backward_workspace_does_not_hold_all_logits(lib):
    n, V, D = 65_536, 131_072, 1024
    assert lib.gt_class_loss_bwd_workspace_size(n, V, D, BF, D, D) < n * V  # a fraction of the 2 n V bytes of bf16
    assert lib.gt_class_loss_fwd_workspace_size(n, V, D, BF, D, D) < n * V // 10


def test_binding_refuses(lib):
    x, w = torch.zeros(4, 8), torch.zeros(5, 8)
    y = torch.zeros(4, dtype=torch.int64)
    rng = torch.zeros(2, dtype=torch.int64)
    for call in (lambda: gt.embed_fwd(w, y), lambda: gt.embed_bwd(y, x, 5), lambda: gt.dropout(x, 0.1, rng),
                 lambda: gt.class_loss_fwd(x, w, y), lambda: gt.class_loss_bwd(x, w, y, y.float(), y.float())):
        with pytest.raises(ValueError):
            call()  # tensors that are not on the GPU
