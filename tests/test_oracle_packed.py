"""CPU pins of the packed-attention, learned-bias and block-norm oracle: hand-worked values, gradients against
differences, and the same results from the full-layer oracle on one sequence."""

import numpy as np
import pytest

from oracle import attention as OA
from oracle import norm as ON
from oracle import packed as OP


def _case(lq, lk, H, Hkv, d, B=0, seed=0):
    rng = np.random.default_rng(seed)
    q_ptr, k_ptr = (np.concatenate([[0], np.cumsum(x)]).astype(np.int64) for x in (lq, lk))
    q, k, v = rng.normal(size=(sum(lq), H, d)), rng.normal(size=(sum(lk), Hkv, d)), rng.normal(size=(sum(lk), Hkv, d))
    do = rng.normal(size=q.shape)
    table = rng.normal(size=(B, H)) if B else None
    _, n = OP.pair_layout(lq, lk)
    ids = rng.integers(0, B + 1, size=n).astype(np.uint8) if B else None
    return q_ptr, k_ptr, q, k, v, do, table, ids


def test_one_sequence_is_the_full_layer():
    q_ptr, k_ptr, q, k, v, do, _, _ = _case([17], [17], 2, 2, 8)
    r, _ = OP.attn(q_ptr, k_ptr, q, k, v, 0.3, dO=do)
    O, L = OA.dense_attn_fwd(q, k, v, 0.3)
    for x, y in zip((r["O"], r["LSE"], r["dQ"], r["dK"], r["dV"]), (O, L) + tuple(OA.dense_attn_bwd(q, k, v, do, 0.3))):
        np.testing.assert_allclose(x, y, rtol=1e-12, atol=1e-12)


def test_causal_by_hand():
    # two queries, three keys: the first query sees keys 0 and 1, the second all; equal scores average the values
    q = np.zeros((2, 1, 1))
    k = np.ones((3, 1, 1))
    v = np.array([1.0, 2.0, 6.0]).reshape(3, 1, 1)
    r, _ = OP.attn([0, 2], [0, 3], q, k, v, 1.0, causal=True)
    np.testing.assert_allclose(r["O"].ravel(), [1.5, 3.0])
    np.testing.assert_allclose(r["LSE"].ravel(), [np.log(2), np.log(3)])
    # more queries than keys: the first ones see nothing
    r, _ = OP.attn([0, 3], [0, 1], np.zeros((3, 1, 1)), k[:1], v[:1], 1.0, causal=True)
    np.testing.assert_allclose(r["O"].ravel(), [0, 0, 1])
    assert list(np.isneginf(r["LSE"].ravel())) == [True, True, False]


@pytest.mark.parametrize("causal", [False, True])
def test_gradients_against_differences(causal):
    lq, lk = [3, 1, 5], [4, 2, 5]
    q_ptr, k_ptr, q, k, v, do, table, ids = _case(lq, lk, 4, 2, 3, B=3, seed=1)

    def loss(q, k, v, table):
        r, _ = OP.attn(q_ptr, k_ptr, q, k, v, 0.7, causal, table, ids)
        return (r["O"] * do).sum()

    r, _ = OP.attn(q_ptr, k_ptr, q, k, v, 0.7, causal, table, ids, dO=do)
    args = [q, k, v, table]
    for n, (name, x) in enumerate(zip(("dQ", "dK", "dV", "dtable"), args)):
        for at in np.ndindex(x.shape):
            step = np.zeros_like(x)
            step[at] = 1e-5
            up, dn = list(args), list(args)
            up[n], dn[n] = x + step, x - step
            assert abs((loss(*up) - loss(*dn)) / 2e-5 - r[name][at]) < 1e-7, (name, at)


def test_bucket_bias_and_gradient_by_hand():
    table = np.array([[1.0, 2.0], [3.0, 4.0]])
    bucket = np.array([1, 0, 2, 1], dtype=np.uint8)
    np.testing.assert_array_equal(OP.bucket_bias(table, bucket), [[3, 4], [1, 2], [-np.inf] * 2, [3, 4]])
    grad = np.arange(8.0).reshape(4, 2)
    np.testing.assert_array_equal(OP.bucket_bias_grad(bucket, grad, 2), [[2, 3], [6, 8]])


@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("gate", ["none", "vector", "rows", "sigmoid"])
def test_norm_gradients_against_differences(layer, gate):
    rng = np.random.default_rng(2)
    n, D = 3, 5
    x, f, dy, dz = (rng.normal(size=(n, D)) for _ in range(4))
    args = dict(x=x, f=f, w_post=rng.normal(size=D), b_post=rng.normal(size=D), w_pre=rng.normal(size=D),
                b_pre=rng.normal(size=D))
    if gate != "none":
        args["gate"] = rng.normal(size=D if gate == "vector" else (n, D))
    fixed = dict(sigmoid=gate == "sigmoid", res_scale=0.6, layer=layer, eps=1e-3)
    r, _ = ON.block(**args, **fixed, dy=dy, dz=dz)

    def loss(**a):
        o, _ = ON.block(**a, **fixed)
        return (o["y"] * dy).sum() + (o["z"] * dz).sum()

    for name, value in args.items():
        for at in np.ndindex(value.shape):
            step = np.zeros_like(value)
            step[at] = 1e-5
            diff = (loss(**{**args, name: value + step}) - loss(**{**args, name: value - step})) / 2e-5
            assert abs(diff - r["d" + name][at]) < 1e-6, (name, at)


def test_norm_by_hand():
    # rms of (3, 4) with eps 0 is sqrt(12.5); y = 2 x + u
    o, _ = ON.block(np.array([[1.0, 1.0]]), np.array([[3.0, 4.0]]), res_scale=2.0, layer=False, eps=0.0)
    np.testing.assert_allclose(o["y"], 2 + np.array([[3.0, 4.0]]) / np.sqrt(12.5))
    np.testing.assert_allclose((o["z"] ** 2).mean(), 1.0)


def _rounded(lq, lk, H, d, dtype, causal, no_d=False, seed=5):
    """One pass with the roundings of the features' type (weights and score gradients where they multiply, O, results;
    fp32 arithmetic for fp32) and D = <dO, O> of the rounded O, or none; and the oracle's."""
    from synth.tensors import bf16_round, normal_tensor

    half, t = (2.0 ** -8, np.float64) if dtype == "bf16" else (2.0 ** -24, np.float32)
    rnd = bf16_round if dtype == "bf16" else (lambda x: x.astype(np.float32))
    q, k, v, do = (normal_tensor((n, H, d), (seed, i), dtype).astype(t) for i, n in enumerate((lq, lk, lk, lq)))
    scale = t(1 / np.sqrt(d))
    ref, _ = OP.attn([0, lq], [0, lk], q, k, v, float(scale), causal, dO=do)
    got = {n: np.zeros(ref[n].shape) for n in ("O", "dQ", "dK", "dV")}
    far = np.arange(lk)[None, :] > np.arange(lq)[:, None] + lk - lq if causal else np.zeros((lq, lk), dtype=bool)
    for h in range(H):
        Q, K, V, G = (x[:, h] for x in (q, k, v, do))
        s = np.where(far, -np.inf, scale * (Q @ K.T))
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        O = got["O"][:, h] = rnd(rnd(p) @ V)
        D = 0 if no_d else (G * O.astype(t)).sum(1, keepdims=True)
        ds = rnd(p * (G @ V.T - D)).astype(t)
        got["dQ"][:, h], got["dK"][:, h] = rnd(scale * (ds @ K)), rnd(scale * (ds.T @ Q))
        got["dV"][:, h] = rnd(rnd(p).astype(t).T @ G)
    return OP.normwise(got, ref, half, max(lq, lk))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lq,lk,d,causal", [(1200, 1200, 64, False), (1200, 1200, 64, True), (700, 2500, 128, True),
                                            (300, 300, 32, False)])
def test_a_backward_without_its_correction_is_outside(dtype, lq, lk, d, causal):
    inside = _rounded(lq, lk, 2, d, dtype, causal)
    assert len(inside) == 4 and max(inside.values()) < 1, inside
    over = _rounded(lq, lk, 2, d, dtype, causal, no_d=True)
    assert over["dQ"] > 1 and over["dK"] > 1, over


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_single_query_without_its_correction_is_outside(dtype):
    assert max(_rounded(1, 9001, 8, 32, dtype, False).values()) < 1
    over = _rounded(1, 9001, 8, 32, dtype, False, no_d=True)
    # dK_j is dS_j q alone: without D it is off by the root of 1 / 9,001 of its size, 0.0105, where bf16 allows 3 * 2^-8
    assert over["dQ"] > 1 and (over["dK"] > 1 or dtype == "bf16"), over
