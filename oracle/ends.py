"""Embedding, dropout and softmax cross entropy over classes in 64 bits, each result with a bound on what fp32
arithmetic and the roundings to the features' type may be off by.

Written with torch's float64 operations, so that the large cases run where their inputs lie; the formulas are elementary
(products, sums, exp) and share no code with the library.

Bounds.  u = 2^-24 is the most that rounding to fp32 moves a value (relative); `half` the same of the features' type.  A
sum of k terms in which each term goes through at most d additions is off by at most d u (sum of the terms' sizes); the
matrix cores' own additions are allowed 2 u.
"""

from __future__ import annotations

import numpy as np
import torch

U = 2.0 ** -24


# ---------------------------------------------------------------------------------------------- embedding

def _terms(ids, n_rows):
    ids = ids.long()
    ids = ids[:, None] if ids.dim() == 1 else ids
    return torch.where((ids >= 0) & (ids < n_rows), ids, n_rows)


def embed(table, ids, scale, half):
    """(out, bound) [n, D] of the scaled sum of the ids' rows."""
    t = table.double()
    t = torch.cat([t, torch.zeros_like(t[:1])])
    rows = t[_terms(ids, table.shape[0])]
    out, size = rows.sum(1) * scale, rows.abs().sum(1) * abs(scale)
    # a field's term goes through at most F additions, then the product with the rounded scale
    return out, (rows.shape[1] + 2) * U * size + half * out.abs()


def embed_grad(ids, dout, n_rows, scale, half, chunk=64, groups=16):
    """(dtable, bound) [R, D].  A row's terms are added in chunks of the sorted pairs, a row's chunks by `groups` lanes."""
    at = _terms(ids, n_rows)
    d = dout.double()
    grad = torch.zeros(n_rows + 1, d.shape[1], dtype=torch.float64, device=d.device)
    size, count = torch.zeros_like(grad), torch.zeros(n_rows + 1, dtype=torch.float64, device=d.device)
    for f in range(at.shape[1]):
        grad.index_add_(0, at[:, f], d)
        size.index_add_(0, at[:, f], d.abs())
        count.index_add_(0, at[:, f], torch.ones(d.shape[0], dtype=torch.float64, device=d.device))
    deep = chunk + torch.ceil(count / chunk / groups) + groups + 2
    grad, size = grad[:-1] * scale, size[:-1] * abs(scale)
    return grad, deep[:-1, None] * U * size + half * grad.abs()


# ------------------------------------------------------------------------------------------------ dropout

def philox(key: int, counter: int, count: int) -> np.ndarray:
    """The words of Philox4x32-10 (Salmon et al., SC 2011) at `count` counters from `counter` on (64 bits of them), as
    uint32 [count, 4]."""
    low = np.uint64(0xFFFFFFFF)
    with np.errstate(over="ignore"):
        c = np.arange(count, dtype=np.uint64) + np.uint64(counter % 2 ** 64)
    x = [c & low, c >> np.uint64(32), np.zeros_like(c), np.zeros_like(c)]
    k = [key % 2 ** 32, (key >> 32) % 2 ** 32]
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k[0]), b & low,
             (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack(x, 1).astype(np.uint32)


def dropout_keep(n: int, p: float, key: int, counter: int) -> np.ndarray:
    """Which of n elements stay."""
    words = philox(key % 2 ** 64, counter, (n + 3) // 4).reshape(-1)[:n]
    return words.astype(np.uint64) >= np.uint64(round(p * 2 ** 32))


def dropout(x, add, keep, p, half):
    """(y, bound)."""
    kept = torch.where(keep, x.double() / (1.0 - p), torch.zeros((), dtype=torch.float64, device=x.device))
    y = kept if add is None else add.double() + kept
    # the factor's rounding, the product's and the sum's
    return y, 2.01 * U * kept.abs() + (0.0 if add is None else U * y.abs()) + half * y.abs()


# --------------------------------------------------------------------------------------------------- loss

def class_loss(x, w, labels, dloss, half, rows=None):
    """{name: (result, bound)} of loss, lse [n], dx [n, D], dw [V, D].  rows: of dW's sum, where these are a part of them
    (the parts' results and bounds then add up, but for the last rounding)."""
    x, w, n, (V, D) = x.double(), w.double(), x.shape[0], w.shape
    y = labels.long()
    has = (y >= 0) & (y < V)
    y = torch.where(has, y, 0)
    wt = w.t().contiguous()
    s = x @ wt
    ds = D * 2 * U * (x.abs() @ wt.abs())  # of the logits
    top = s.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(s - top).sum(1, keepdim=True))
    p = torch.exp(s - lse)
    # of lse: the logits', the exponents' (a difference, a rounded constant and a product), exp's own, the sums' (a
    # lane's 64 classes, then the blocks' results, each scaled once), the logarithm's and the last sum's; the loss is
    # the largest logit's distance from the label's and the same logarithm, and no rounding of lse's size
    blocks = -(-V // 64)
    dsum = (1.01 * (p * ds).sum(1, keepdim=True) + 4 * U * (p * (top - s)).sum(1, keepdim=True)
            + U * (90 + 3 * blocks) + 4 * U * (lse - top))
    dlse = dsum + 2 * U * lse.abs()
    at = torch.arange(n, device=x.device)
    sy, dsy = s[at, y], ds[at, y]
    loss = lse[:, 0] - sy
    out = {"lse": (torch.where(has, lse[:, 0], 0.0), dlse[:, 0]),
           "loss": (torch.where(has, loss, 0.0), dsum[:, 0] + dsy + 2 * U * (loss + top[:, 0] - sy))}
    up = torch.where(has, dloss.double(), 0.0)[:, None]
    dp = 1.01 * p * (ds + dlse + 4 * U * (s - lse).abs() + 4 * U)
    g = p
    g[at, y] -= 1.0
    g = g * up
    # of dL: p's and the subtraction's roundings, four more of factors (dloss over its largest, the product, the largest
    # again at the end), then the rounding to the features' type
    dg = up.abs() * (dp + U) + 5 * U * g.abs() + half * g.abs()
    del s, ds, p, dp
    dx, dw = g @ w, g.t().contiguous() @ x
    out["dx"] = dx, dg @ w.abs() + 2 * U * V * (g.abs() @ w.abs()) + half * dx.abs()
    gt, dgt = g.abs().t().contiguous(), dg.t().contiguous()
    out["dw"] = dw, dgt @ x.abs() + 2 * U * (rows or n) * (gt @ x.abs()) + half * dw.abs()
    return out
