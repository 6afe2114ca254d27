"""The class loss's workspaces stay within what their arrays are said to take (no GPU): the logits' gradient is held a
piece at a time, for many rows as for many classes."""

import os

import pytest

from paper_2407_14106_amd import gt

MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gt.LIB_PATH):
        from paper_2407_14106_amd import build

        build.build()
    return gt.load_library()


@pytest.mark.parametrize("dt,size", [(gt.GT_BF16, 2), (gt.GT_F32, 4)])
@pytest.mark.parametrize("D", [16, 64, 256, 1024])
def test_backward_holds_a_piece_of_the_logits_gradient(lib, D, dt, size):
    for n in (100_000, 131_072, 131_073, 400_000, 1_000_000, 2_000_000):
        for V in (2, 47, 172, 600, 1000, 1024, 1025, 2000, 128_000):
            holds_a_piece(lib, n, V, D, dt, size)


def holds_a_piece(lib, n, V, D, dt, size):
    need = lib.gt_class_loss_bwd_workspace_size(n, V, D, dt, D, D)
    # a piece's dL both ways round, of 1 GB each where 1,024 classes or all of fewer are a piece, rounded up to whole
    # blocks of 256 a side and with 64 elements behind a row of 4 KB and more
    classes = min(-(-V // 64) * 64, 1024)
    rows = min(n, 1024 * MB // (classes * size)) + 256
    piece = 2 * size * (rows + 64) * (classes + (256 if V > 64 else 0) + (64 if classes * size >= 4096 - 256 else 0))
    # X the other way round, and in order (more than 2,048 classes, or rows off their alignment); a piece of W the same
    row = -(-D * size // 128) * 128
    turned = row * (n + 512) * (2 if V > 2048 or row != D * size else 1) + row * (V if row != D * size else 0)
    turned += size * D * (min(V, 1024) + 512)
    sums = 4 * n * D if V > 1024 else 0
    # the list, and the parts of split sums: of 256 CUs, five blocks of 64 x 64 or one of 256 x 256 each, twice
    rest = 4 * n + MB + 2 * 256 * 256 * 256 * 4 + 4 * D * 1280
    assert need <= piece + turned + sums + rest, (n, V)
    if n * V * size > 4000 * MB:
        assert need - turned - sums < n * V * size, (n, V)  # a part of the logits


def test_backward_of_a_million_rows(lib):
    # 47 and 1,000 classes: with a gradient of all rows and 256 classes at least 1.8, 4.4 and 8.7 GB
    need = lib.gt_class_loss_bwd_workspace_size
    assert need(1_000_000, 47, 256, gt.GT_BF16, 256, 256) < 850 * MB  # of which X the other way round is 488
    assert need(1_000_000, 1000, 64, gt.GT_BF16, 64, 64) < 2_300 * MB
    assert need(1_000_000, 1000, 64, gt.GT_F32, 64, 64) < 2_400 * MB
