"""Softmax attention inside packed sequences, in fp64, written out head by head.

Oracle - test infrastructure only (see the package docstring).

Sequence s holds the queries q_ptr[s]..q_ptr[s+1]-1 and the keys
k_ptr[s]..k_ptr[s+1]-1, lq and lk of them.  Its query i attends to its key j
unless (causal) j > i + lk - lq, or (with a learned bias) the pair's bucket is
not in the table.  Query head h reads kv head h // (H / Hkv):

    s_ij = scale <Q[i,h], K[j,h']> + table[bucket_ij, h]
    LSE_i = log sum_j exp(s_ij)          (-inf where nothing is attended to)
    P_ij = exp(s_ij - LSE_i),  O[i,h] = sum_j P_ij V[j,h']
    dP_ij = <dO[i,h], V[j,h']>,  D_i = sum_j P_ij dP_ij,  dS_ij = P_ij (dP_ij - D_i)
    dQ[i,h] = scale sum_j dS_ij K[j,h'],  dK[j,h'] = scale sum_{i, h of h'} dS_ij Q[i,h]
    dV[j,h'] = sum_{i, h of h'} P_ij dO[i,h],  dtable[b,h] = sum_{bucket_ij = b} dS_ij

Buckets are bytes: sequence after sequence a row of lk for each query, padded
to a multiple of 16.

``bounds`` gives beside each result how far a computation may be off that forms
dot products and sums in fp32 in any order, rounds weights and score gradients
to the features' type where they multiply a row, and rounds results once.
"""

from __future__ import annotations

import numpy as np


def pair_layout(lq, lk):
    """First byte of each sequence's buckets, and the number of bytes."""
    wide = [(b + 15) // 16 * 16 for b in lk]
    at = np.concatenate([[0], np.cumsum([a * w for a, w in zip(lq, wide)])]).astype(np.int64)
    return at[:-1], int(at[-1])


def pair_buckets(buckets, lq, lk, s):
    """The [lq, lk] buckets of sequence s."""
    at, _ = pair_layout(lq, lk)
    wide = (lk[s] + 15) // 16 * 16
    return buckets[at[s]:at[s] + lq[s] * wide].reshape(lq[s], wide)[:, :lk[s]].astype(np.int64)


def _heads(q_ptr, k_ptr, H, Hkv):
    for s in range(len(q_ptr) - 1):
        for h in range(H):
            yield s, h, h // (H // Hkv), slice(q_ptr[s], q_ptr[s + 1]), slice(k_ptr[s], k_ptr[s + 1])


def _scores(s, h, q, k, scale, causal, table, ids):
    """Scores [lq, lk], -inf where not attended to."""
    lq, lk = q.shape[0], k.shape[0]
    sc = scale * (q @ k.T)
    if causal:
        i, j = np.arange(lq)[:, None], np.arange(lk)[None, :]
        sc = np.where(j <= i + lk - lq, sc, -np.inf)
    if table is not None:
        B = table.shape[0]
        sc = np.where(ids < B, sc + table[np.minimum(ids, B - 1), h], -np.inf)
    return sc


def _softmax(sc):
    if sc.shape[1] == 0:
        return sc, np.full(sc.shape[0], -np.inf)
    m = sc.max(axis=1)
    ref = np.where(np.isfinite(m), m, 0.0)
    e = np.exp(sc - ref[:, None])
    total = e.sum(axis=1)
    with np.errstate(divide="ignore"):
        lse = ref + np.log(total)
    return e / np.where(total > 0, total, 1.0)[:, None], lse


def attn(q_ptr, k_ptr, Q, K, V, scale, causal=False, table=None, buckets=None, dO=None, half=2.0 ** -24,
         exact_d=True):
    """A dict of results O, LSE (and with dO: dQ, dK, dV, dtable), and a dict of bounds for the same names.

    half: the features' half step (2**-8 for bf16, 2**-24 for fp32).  exact_d: D is formed from the scores; else as
    <dO, O> from an O that is itself off by its bound."""
    Q, K, V = (np.asarray(x, dtype=np.float64) for x in (Q, K, V))
    dO = None if dO is None else np.asarray(dO, dtype=np.float64)
    table = None if table is None else np.asarray(table, dtype=np.float64)
    nq, H, d = Q.shape
    nk, Hkv = K.shape[:2]
    lq, lk = np.diff(q_ptr), np.diff(k_ptr)
    u = 2.0 ** -24  # fp32's half step
    r = {"O": np.zeros_like(Q), "LSE": np.full((nq, H), -np.inf)}
    b = {"O": np.zeros_like(Q), "LSE": np.zeros((nq, H))}
    if dO is not None:
        for name, x in (("dQ", Q), ("dK", K), ("dV", V)):
            r[name], b[name] = np.zeros_like(x), np.zeros_like(x)
        if table is not None:
            r["dtable"], b["dtable"] = np.zeros(table.shape), np.zeros(table.shape)
    for s, h, hk, qs, ks in _heads(q_ptr, k_ptr, H, Hkv):
        if qs.start == qs.stop or ks.start == ks.stop:
            continue
        q, k, v = Q[qs, h], K[ks, hk], V[ks, hk]
        ids = None if table is None else pair_buckets(buckets, lq, lk, s)
        sc = _scores(s, h, q, k, scale, causal, table, ids)
        p, lse = _softmax(sc)
        n = k.shape[0]
        # a score: d + 4 roundings of its terms (and of the bias); a weight: its score's and its reference's, the
        # exponential's and its argument's, and the sum's n additions
        live = np.where(np.isfinite(sc), np.abs(sc), 0.0)
        e_s = (d + 4) * u * (abs(scale) * (np.abs(q) @ np.abs(k).T)) + 4 * u * live
        e_row = e_s.max(axis=1, initial=0.0)[:, None]
        # an fp32 score or statistic of size |s| is itself a rounded number
        w = 2 * (e_s + e_row) + (n + 16) * u + 4 * u * live.max(axis=1, initial=0.0)[:, None]
        r["O"][qs, h], r["LSE"][qs, h] = p @ v, lse
        b["O"][qs, h] = ((half + w + n * u) * p) @ np.abs(v) + half * np.abs(p @ v)
        b["LSE"][qs, h] = 2 * e_row[:, 0] + (n + 16) * u + 4 * u * np.where(np.isfinite(lse), np.abs(lse), 0.0)
        if dO is None:
            continue
        g = dO[qs, h]
        dp = g @ v.T
        D = (p * dp).sum(axis=1, keepdims=True)
        ds = p * (dp - D)
        e_dp = (d + 4) * u * (np.abs(g) @ np.abs(v).T)
        if exact_d:
            e_d = ((w + n * u) * p * np.abs(dp) + p * e_dp).sum(axis=1, keepdims=True)
        else:
            e_d = (np.abs(g) * b["O"][qs, h]).sum(axis=1, keepdims=True) + d * u * np.abs(g * r["O"][qs, h]).sum(
                axis=1, keepdims=True)
        e_ds = w * np.abs(ds) + p * (e_dp + e_d + 2 * u * (np.abs(dp) + np.abs(D)))
        rows = q.shape[0] * (H // Hkv)
        r["dQ"][qs, h] = scale * (ds @ k)
        b["dQ"][qs, h] = abs(scale) * ((e_ds * (1 + half) + (half + n * u) * np.abs(ds)) @ np.abs(k))
        r["dK"][ks, hk] += scale * (ds.T @ q)
        b["dK"][ks, hk] += abs(scale) * ((e_ds * (1 + half) + (half + rows * u) * np.abs(ds)).T @ np.abs(q))
        r["dV"][ks, hk] += p.T @ g
        b["dV"][ks, hk] += ((half + w + rows * u) * p).T @ np.abs(g)
        if table is not None:
            for x in range(table.shape[0]):
                at = ids == x
                r["dtable"][x, h] += ds[at].sum()
                b["dtable"][x, h] += e_ds[at].sum() + min(at.sum(), 4096) * u * np.abs(ds[at]).sum()
    for name in ("dQ", "dK", "dV"):
        if name in r:
            b[name] += 2 * half * np.abs(r[name])
    if "dtable" in r:
        b["dtable"] += 2 * u * np.abs(r["dtable"])
    return r, b


def bucket_bias(table, bucket):
    """The per-edge bias: the table's rows, -inf for a bucket that is not in it."""
    B = table.shape[0]
    return np.where((bucket < B)[:, None], table[np.minimum(bucket.astype(np.int64), B - 1)], -np.inf)


def bucket_bias_grad(bucket, dbias, B):
    """dtable[b] = the sum of dbias over the edges of bucket b."""
    out = np.zeros((B, dbias.shape[1]))
    for b in range(B):
        out[b] = dbias[bucket == b].astype(np.float64).sum(axis=0)
    return out


def normwise(got, ref, half, most):
    """The error of O, dQ, dK and dV as whole arrays over their tolerance (above 1 is outside): the elementwise bounds
    add a row's terms as absolute values, which for rows of hundreds of partners is a large part of the result.

    A half step for the weights or score gradients where they multiply, one for the result, and one for what a rounded O
    does to D (which moves a gradient by less than that of its size: it is multiplied by a mean of K or Q, smaller than
    the gradient by the root of the partners' number).  In fp32 besides, over rows of at most `most` partners and d
    features: 4 (most + d) half steps of 2^-24 for the sums and the scores."""
    out = {}
    for name in ("O", "dQ", "dK", "dV"):
        if name in ref:
            r = ref[name]
            tol = 3 * half + 4 * (most + r.shape[2]) * 2.0 ** -24
            out[name] = float(np.linalg.norm(np.asarray(got[name], dtype=np.float64) - r) / (tol * np.linalg.norm(r)))
    return out
