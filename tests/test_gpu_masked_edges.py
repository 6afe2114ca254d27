"""GPU sparse attention whose bias takes edges out (-inf, as the learned bias gives for a bucket that the table does
not hold), whole rows and columns among them, and rows without edges beside others in a dense tile: forward, the
gradients, dB and the table's gradient vs the fp64 oracle on the edges that are left, head by head."""

import sys

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import packed as OP
from synth import csr_from_pairs
from synth.tensors import normal_tensor
from tests.helpers import assert_close, dev_csr, dev_feat, grad_term_rms, host

pytestmark = pytest.mark.gpu

CSR_ONLY = 1_000_001  # no dense tile: every edge on the edge kernels
PLANS = [(128, CSR_ONLY), (128, 0), (64, 0), (128, 50_000)]
HUB, LONG = 5, 650  # nodes of more edges than GT_LONG_ROW: one that attends to nothing, one that keeps its edges


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def graph(n=700):
    rng = np.random.default_rng(3)
    u, v = rng.integers(0, n, size=9 * n), rng.integers(0, n, size=9 * n)
    near = np.arange(n).repeat(12)
    w = np.clip(near + rng.integers(-20, 21, size=len(near)), 0, n - 1)
    hubs = [np.repeat(x, 400) for x in (HUB, LONG)]
    ends = [rng.permutation(n)[:400] for _ in hubs]
    return csr_from_pairs(n, np.concatenate([u, near, *hubs, *ends]), np.concatenate([v, w, *ends, *hubs]),
                          symmetric=False, self_loops=False)


def reference(rowptr, col, q, k, v, do, scale, bias):
    """O, LSE, dQ, dK, dV, dB: each head's oracle on the edges that its bias leaves."""
    n, H, _ = q.shape
    rows = np.repeat(np.arange(n), np.diff(rowptr))
    out = [np.zeros(q.shape), np.full((n, H), -np.inf), *(np.zeros(q.shape) for _ in range(3)), np.zeros(bias.shape)]
    for h in range(H):
        keep = np.isfinite(bias[:, h])
        rp = np.concatenate([[0], np.cumsum(np.bincount(rows[keep], minlength=n))])
        args = (rp, col[keep], *(x[:, h:h + 1] for x in (q, k, v)))
        out[0][:, h:h + 1], out[1][:, h:h + 1] = OA.sparse_attn_fwd(*args, scale, bias=bias[keep, h:h + 1])
        dq, dk, dv, db = OA.sparse_attn_bwd(*args, do[:, h:h + 1], scale, bias=bias[keep, h:h + 1])
        out[2][:, h:h + 1], out[3][:, h:h + 1], out[4][:, h:h + 1], out[5][keep, h:h + 1] = dq, dk, dv, db
    return out


def compare(gt, rowptr, col, H, d, dtype, table, ids, T, tau, seed, odd=False):
    say("masked edges", len(rowptr) - 1, len(col), H, d, dtype, T, tau, odd)
    n, scale = len(rowptr) - 1, 1.0 / np.sqrt(d)
    q, k, v, do = (normal_tensor((n, H, d), (seed, t), dtype) for t in range(4))
    bias = OP.bucket_bias(table.astype(np.float64), ids)
    rp, cl = dev_csr(rowptr, col)
    Q, K, V, dO = (dev_feat(x, dtype) for x in (q, k, v, do))
    if odd:  # features off a multiple of 16 bytes
        shift = lambda x: torch.cat([x.new_zeros(1), x.reshape(-1)])[1:].view(x.shape)  # noqa: E731
        Q, K, V, dO = (shift(x) for x in (Q, K, V, dO))
    I = torch.from_numpy(ids).cuda()
    plan = gt.build_tiles(rp, cl, T, tau, edge_positions=True)
    assert (plan.n_dense > 0) == (tau != CSR_ONLY)
    b = gt.bucket_bias_fwd(torch.from_numpy(table).cuda(), I)
    O, L = gt.sparse_attn_fwd_bias(plan, Q, K, V, b, scale)
    dQ, dK, dV, dB = gt.sparse_attn_bwd_bias(plan, gt.edge_map(plan), Q, K, V, b, dO, L, scale)
    dT = gt.bucket_bias_bwd(I, dB, len(table))
    torch.cuda.synchronize()
    ref = reference(rowptr, col, q, k, v, do, scale, bias)
    floors = (None, None) + grad_term_rms(rowptr, col, q, k, v, do, scale)
    for name, x, r, rho in zip(("O", "LSE", "dQ", "dK", "dV", "dB"), (O, L, dQ, dK, dV, dB), ref, floors):
        assert_close(host(x), r, dtype, name, rho=rho)
    assert (host(dB)[~np.isfinite(bias)] == 0).all()
    # the edges' own tolerance, summed over each bucket's edges
    each = 2e-2 + 1e-2 * np.abs(ref[5]) if dtype == "bf16" else 1e-5 * np.maximum(max(1.0, floors[5]), np.abs(ref[5]))
    over = np.abs(host(dT) - OP.bucket_bias_grad(ids, ref[5], len(table))) - OP.bucket_bias_grad(ids, each, len(table))
    assert over.max() <= 0, f"dtable: outside its bound by up to {over.max():.3e}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,d", [(1, 64), (2, 32), (4, 32), (8, 64), (16, 32)])
@pytest.mark.parametrize("T,tau", PLANS)
def test_rows_and_columns_that_the_bias_takes_out(gt, dtype, H, d, T, tau):
    rowptr, col = graph()
    n, B = len(rowptr) - 1, 7
    rng = np.random.default_rng(H + d)
    rows = np.repeat(np.arange(n), np.diff(rowptr))
    ids = rng.integers(0, B, size=len(col)).astype(np.uint8)
    ids[rng.random(len(col)) < 0.1] = 200
    ids[np.isin(rows, [0, HUB, 64, 65, 127, 128, 333, n - 1])] = 255  # these attend to nothing
    ids[np.isin(col, [1, 2, 300, n - 2])] = B  # nobody attends to these
    table = rng.normal(size=(B, H)).astype(np.float32)
    table[3, 0] = -np.inf  # a bucket out for one head
    compare(gt, rowptr, col, H, d, dtype, table, ids, T, tau, seed=H + d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,tau", PLANS)
def test_every_edge_taken_out(gt, dtype, T, tau):
    rowptr, col = graph()
    table = np.ones((3, 4), dtype=np.float32)
    compare(gt, rowptr, col, 4, 32, dtype, table, np.full(len(col), 3, dtype=np.uint8), T, tau, seed=1)


@pytest.mark.parametrize("T", [64, 128])
def test_features_at_any_address(gt, T):
    # bf16 features off a multiple of 16 bytes take the general matrix-core tiles
    rowptr, col = graph()
    rows = np.repeat(np.arange(len(rowptr) - 1), np.diff(rowptr))
    ids = np.where(rows % 9 == 0, 255, rows % 4).astype(np.uint8)
    table = np.random.default_rng(0).normal(size=(4, 4)).astype(np.float32)
    compare(gt, rowptr, col, 4, 64, "bf16", table, ids, T, 0, seed=2, odd=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [64, 128])
def test_rows_without_edges_inside_a_dense_tile(gt, dtype, T):
    # a bias on every edge, none of them out: nodes 40 to 49 have no edges, in a tile whose other rows have
    rng = np.random.default_rng(6)
    u, v = rng.integers(0, 300, size=4000), rng.integers(0, 300, size=4000)
    keep = (u < 40) | (u > 49)
    rowptr, col = csr_from_pairs(300, u[keep], v[keep], symmetric=False, self_loops=False)
    table = rng.normal(size=(5, 8)).astype(np.float32)
    compare(gt, rowptr, col, 8, 32, dtype, table, rng.integers(0, 5, size=len(col)).astype(np.uint8), T, 0, seed=4)
