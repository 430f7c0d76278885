"""fp64 CPU oracle for the losses over the tokens of sequences (see include/eexit.h, "Losses over the tokens of sequences").

TEST INFRASTRUCTURE ONLY (see oracle/exit_head.py).  Shares no code with the CUDA sources.
"""
from __future__ import annotations

import numpy as np


def _slices(seq_start, M):
    s = [min(max(int(v), 0), M) for v in seq_start]
    return [slice(a, max(a, b)) for a, b in zip(s[:-1], s[1:])]


def policy_loss(ce, old_ce, adv, labels, V, ref_ce=None, kl_weight=0.0, clip=(0.2, 0.2), seq_start=None) -> dict:
    """loss [4] (total, policy, kl, share of tokens the clamp decided), dce [M]."""
    ce, old_ce, adv = (np.asarray(x, dtype=np.float64) for x in (ce, old_ce, adv))
    M = ce.size
    counted = (labels >= 0) & (labels < V)
    loss, dce = np.zeros(4), np.zeros(M)
    units = [slice(0, M)] if seq_start is None else _slices(seq_start, M)
    for u, rows in enumerate(units):
        at = np.flatnonzero(counted[rows]) + rows.start
        if at.size == 0:
            continue
        w = 1.0 / (at.size * len(units))
        a = adv[at] if seq_start is None else adv[u]
        x = old_ce[at] - ce[at]
        r = np.exp(x)
        # clamped where the clamped value is the smaller one
        cut = np.where(a > 0, x > np.log1p(clip[1]), (a < 0) & (x < np.log1p(-clip[0])))
        policy = -a * np.where(cut, np.where(a > 0, 1.0 + clip[1], 1.0 - clip[0]), r)
        g = np.where(cut, 0.0, a * r)
        kl = np.zeros(at.size)
        if ref_ce is not None:
            gap = ce[at] - np.asarray(ref_ce, dtype=np.float64)[at]
            kl = np.expm1(gap) - gap
            g = g + kl_weight * np.expm1(gap)
        loss += w * np.array([(policy + kl_weight * kl).sum(), policy.sum(), kl.sum(), cut.sum()])
        dce[at] = w * g
    return dict(loss=loss, dce=dce)


def preference_loss(ce, labels, V, seq_start, ref_ce=None, beta=0.1, smoothing=0.0) -> dict:
    """loss [4] (mean, share of positive margins, rewards of the preferred and the rejected), margin [P], dce [M]."""
    ce = np.asarray(ce, dtype=np.float64)
    M = ce.size
    counted = (labels >= 0) & (labels < V)
    ref = np.zeros(M) if ref_ce is None else np.asarray(ref_ce, dtype=np.float64)
    gain = np.zeros(M)
    gain[counted] = ref[counted] - ce[counted]
    units = _slices(seq_start, M)
    reward = beta * np.array([gain[u].sum() for u in units])
    good, bad = reward[0::2], reward[1::2]
    m = good - bad
    P = m.size
    up, down = np.logaddexp(0.0, -m), np.logaddexp(0.0, m)
    slope = (smoothing * np.exp(-up) - (1.0 - smoothing) * np.exp(-down)) / P
    dce = np.zeros(M)
    for p in range(P):
        dce[units[2 * p]] = -beta * slope[p]
        dce[units[2 * p + 1]] = beta * slope[p]
    loss = np.array([((1.0 - smoothing) * up + smoothing * down).mean(), (m > 0).mean(), good.mean(), bad.mean()])
    return dict(loss=loss, margin=m, dce=np.where(counted, dce, 0.0))
