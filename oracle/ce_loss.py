"""fp64 CPU oracle for the supervised objective of a head and its gradient (paper section 3.3, "Losses": L_CE).

TEST INFRASTRUCTURE ONLY (see oracle/exit_head.py).  Shares no code with the CUDA sources.

Per token: y = LayerNorm(h) rounded to fp32 and then to bf16, z = W y, lse = ln sum exp z, ce = lse - z[label].  Rows whose label is
outside [0, V) are not counted.  Gradient of sum_i w_i ce_i, the rounding of y passed through:
    g = w (softmax(z) - onehot(label)),  dy = g W,  dW = g^T y,
    t = dy * gamma,  dh = rstd (t - mean t - xhat mean(t xhat)),  dgamma = sum dy xhat,  dbeta = sum dy.

Pins (tests/test_oracle_ce.py): closed forms, central differences of the loss in every input, rows not counted.
"""
from __future__ import annotations

import numpy as np

from .exit_head import bf16_decode, bf16_rne


def bf16_by_f32(x):
    """fp64 -> fp32 -> bf16, each to nearest: what casting a LayerNorm that returns fp32 gives."""
    return bf16_rne(np.asarray(x, dtype=np.float64).astype(np.float32).astype(np.float64))


def _rows(h_bits, head):
    x = bf16_decode(h_bits)
    c = x - x.mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt((c * c).mean(axis=1, keepdims=True) + head["ln_eps"])
    xhat = c * rstd
    return xhat, rstd, xhat * head["gamma"].astype(np.float64) + head["beta"].astype(np.float64)


def cross_entropy(h_bits, head, labels, weights=None, round_y: bool = True) -> dict:
    """ce, lse [M], loss (mean over counted rows), n; and the gradient dh, dW, dgamma, dbeta of sum_i weights_i ce_i
    (weights None: of the mean).  Also the intermediate values a tolerance is made of: y, P = softmax, G, dy, xhat, rstd."""
    labels = np.asarray(labels)
    W = bf16_decode(head["W"])
    V = W.shape[0]
    M = h_bits.shape[0]
    counted = (labels >= 0) & (labels < V)
    xhat, rstd, y = _rows(h_bits, head)
    if round_y:
        y = bf16_by_f32(y)
    z = y @ W.T
    top = z.max(axis=1, keepdims=True)
    P = np.exp(z - top)
    total = P.sum(axis=1, keepdims=True)
    lse = (top + np.log(total))[:, 0]
    P /= total
    at = np.where(counted, labels, 0)
    ce = np.where(counted, lse - z[np.arange(M), at], 0.0)
    n = int(counted.sum())
    w = np.full(M, 1.0 / max(n, 1)) if weights is None else np.asarray(weights, dtype=np.float64)
    w = np.where(counted, w, 0.0)
    live = w != 0.0
    G = np.where(live[:, None], P, 0.0)
    G[np.flatnonzero(live), at[live]] -= 1.0
    G *= w[:, None]
    y_live = np.where(live[:, None], y, 0.0)
    dy = G @ W
    t = dy * head["gamma"].astype(np.float64)
    xhat_live = np.where(live[:, None], xhat, 0.0)
    dh = rstd * (t - t.mean(axis=1, keepdims=True) - xhat_live * (t * xhat_live).mean(axis=1, keepdims=True))
    dh = np.where(live[:, None], dh, 0.0)
    return dict(ce=ce, lse=lse, loss=float(ce.sum() / max(n, 1)), n=n, dh=dh, dW=G.T @ y_live, dgamma=(dy * xhat_live).sum(axis=0),
                dbeta=dy.sum(axis=0), y=y, P=P, G=G, W=W, dy=dy, xhat=xhat_live, rstd=rstd, weights=w)
