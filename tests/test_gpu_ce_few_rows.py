"""The gradient of ee_head_ce where one entry of the logits' gradient G, the label's, outweighs the others: its rounding to bf16, which all of a
row would share, must not reach dh, dgamma and dbeta.

Bounds: those of test_gpu_ce.py without the rounding of the label's entry of G, for which 4u of its magnitude stand (its own fp32
arithmetic, and what is left of it after the rounding, times W, added to dy).  The other entries are rounded: e = 2^-8 of each.  The weight rows of the labels are 16
times as long as the others, so that what those roundings can do is small next to it.
"""
import numpy as np
import pytest
import torch

import gen
import oracle
from _util import dev, dev_bf16
from test_gpu_ce import E, U, _np, bounds

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _case(M, d, V):
    rng = np.random.default_rng(M + d + V)
    W = rng.normal(0, 0.02, (V, d))
    labels = rng.choice(V, M, replace=M > V).astype(np.int32)
    labels[0] = V - 1
    W[labels] = rng.normal(0, 0.32, (M, d))
    head = dict(gamma=np.full(d, 0.05, np.float32), beta=rng.normal(0, 0.01, d).astype(np.float32), W=gen.bf16_bits_from_f32(W.astype(np.float32)), ln_eps=1e-5)
    return gen.bf16_bits_from_f32(rng.normal(0, 1, (M, d)).astype(np.float32)), head, labels


def _bounds(ref, gamma, labels, counted):
    """bounds() with the label's |G| taken out of its rounding term: the same formulas with E |G| replaced, for what comes through dy."""
    M, V = ref["G"].shape
    d = ref["W"].shape[1]
    y, W, P, w = ref["y"], ref["W"], ref["P"], np.abs(ref["weights"])
    dz = 2 * U * d * (np.abs(y) @ np.abs(W).T).max(axis=1)
    dlse = dz + 2.0 ** -21 + 2 * U * (64 + V / 64) + 2 * U * np.abs(ref["lse"])
    r = dz + dlse + 2.0 ** -21
    rounded = np.abs(ref["G"]).copy()
    rows = np.flatnonzero(counted)
    rounded[rows, labels[rows]] *= 4 * U / E
    dG = (w * r)[:, None] * P * (1 + E) + E * rounded * (1 + U * 8)
    aG = np.abs(ref["G"])
    Ddy = dG @ np.abs(W) + 2 * U * (V + 40) * (aG @ np.abs(W))
    g, x, s = np.abs(gamma).astype(np.float64), np.abs(ref["xhat"]), ref["rstd"]
    t = np.abs(ref["dy"]) * g
    Dt = Ddy * g + 4 * U * t
    inner = Dt + Dt.mean(1, keepdims=True) + x * (Dt * x).mean(1, keepdims=True)
    size = t + t.mean(1, keepdims=True) + x * (t * x).mean(1, keepdims=True)
    dh = s * (inner + 2 * U * (d + 16) * size + 8 * U * (x + 4.0) * (t * (x + 1)).mean(1, keepdims=True))
    adds = 2 * U * (M + 16)
    out = dict(dh=dh * (1 + E) + E * np.abs(ref["dh"]) + 1e-38)
    out["dgamma"] = ((Ddy * x).sum(0) + adds * (np.abs(ref["dy"]) * (x + 4.0)).sum(0)) * (1 + E) + E * np.abs(ref["dgamma"]) + 1e-38
    out["dbeta"] = (Ddy.sum(0) + adds * np.abs(ref["dy"]).sum(0)) * (1 + E) + E * np.abs(ref["dbeta"]) + 1e-38
    return out


@pytest.mark.parametrize("M,d,V", [(1, 64, 5000), (2, 128, 3001), (16, 64, 2000), (64, 520, 3000), (130, 264, 4000), (40, 6000, 600), (300, 72, 50304)])
@pytest.mark.parametrize("weighted", [False, True])
def test_the_label_of_a_row_is_not_rounded_for_all_of_it(ee, M, d, V, weighted):
    h_bits, head, labels = _case(M, d, V)
    if M > 4:
        labels[3::5] = -1
    rng = np.random.default_rng(2)
    weights = rng.normal(0, 1, M).astype(np.float32) if weighted else None
    if weighted and M > 4:
        weights[1] = 0.0
    ref = oracle.cross_entropy(h_bits, head, labels, weights)
    bnd = _bounds(ref, head["gamma"], labels, labels >= 0)
    dhead = dict(h=dev_bf16(h_bits), gamma=dev(head["gamma"]), beta=dev(head["beta"]), W=dev_bf16(head["W"]))
    ws = ee.new_head_ce_grad_workspace(M, d, V)
    fwd = ee.ee_head_ce(dhead, dev(labels), 1e-5, workspace=ws)
    ws[256:256 + (ws.numel() - 256) // 4 * 4].view(torch.float32).fill_(float("nan"))
    got = ee.ee_head_ce_grad(dhead, dev(labels), 1e-5, fwd, dce=None if weights is None else dev(weights), workspace=ws)
    for k in bnd:
        err = np.abs(_np(got[k]) - ref[k])
        worst = np.unravel_index(np.argmax(err / bnd[k]), err.shape)
        assert np.all(err <= bnd[k]), (k, worst, err[worst], bnd[k][worst], ref[k][worst])
    full = bounds(ref, head["gamma"])
    assert (np.abs(_np(got["dW"]) - ref["dW"]) <= full["dW"]).all()
