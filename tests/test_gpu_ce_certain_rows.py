"""ee_head_ce on rows that are nearly certain of their token: the loss is then far below a step of lse in fp32.

With m the row's largest logit, ce = (m - z_label) + ln(1 + r), r = sum over the other logits of exp(z - m).  Bound, u = 2^-24:
  a logit is off by at most dz = 2 u d max_v sum_j |w_vj y_j| (as in test_gpu_ce.py), a difference of two by 2 dz, and its rounding and that
  of its product with log2 e by 2u |z - m|, which matters only for terms above 2^-126, |z - m| <= 88;
  r   relative: x = 2 dz + 2u 88 + 2^-21 (the exponential) + 2u (64 + V / 64) (additions and rescalings)
  ce  x ln(1 + r) + 2u ce, and where the label is not the largest logit 2 dz more
"""
import numpy as np
import pytest
import torch

import gen
import oracle
from _util import dev, dev_bf16
from test_gpu_ce import E, _np

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _case(M, d, V, seed, twins=False):
    """Rows that lean towards a weight row each, from hardly to so strongly that their loss is 1e-8."""
    rng = np.random.default_rng(seed)
    w_bits = gen.bf16_bits_from_f32(rng.normal(0, 2.0 / np.sqrt(d), (V, d)).astype(np.float32))
    if twins:                                                            # every weight row once more, in another tile: two largest logits
        w_bits[V // 2:V // 2 * 2] = w_bits[:V // 2]
    W = oracle.bf16_decode(w_bits)
    token = rng.integers(0, V, M)
    token[0], token[-1] = V - 1, 0
    pull = W[token] / np.linalg.norm(W[token], axis=1, keepdims=True) * np.sqrt(d)
    lean = np.linspace(0.2, 1.0, M)[:, None] if M > 1 else np.ones((1, 1))
    h_bits = gen.bf16_bits_from_f32((lean * pull + (1 - lean) * rng.normal(0, 1, (M, d))).astype(np.float32))
    gamma, beta = np.full(d, 14.0 / np.sqrt(d), np.float32), np.zeros(d, np.float32)      # logits of the tokens up to 28
    labels = token.astype(np.int32)
    labels[2::7] = (labels[2::7] + 1) % V                                # some rows are certain of another token
    labels[5::11] = -1
    return h_bits, dict(gamma=gamma, beta=beta, W=w_bits, ln_eps=1e-5), labels


SIZES = [(1, 64, 200), (40, 64, 200), (64, 128, 3001), (128, 256, 5000), (150, 128, 2500), (700, 64, 1500), (1100, 64, 1003)]


@pytest.mark.parametrize("M,d,V", SIZES)
@pytest.mark.parametrize("twins", [False, True])
def test_the_loss_of_nearly_certain_rows_keeps_its_digits(ee, M, d, V, twins):
    h_bits, head, labels = _case(M, d, V, M + d + V, twins)
    ref = oracle.cross_entropy(h_bits, head, labels)
    W = ref["W"]
    z = ref["y"] @ W.T
    top = z.argmax(1)
    m = z.max(1)
    e = np.exp(z - m[:, None])
    e[np.arange(M), top] = 0.0                                           # the others; in 64 bits the sum keeps its digits
    rest = np.log1p(e.sum(1))
    counted = labels >= 0
    at = np.where(counted, labels, 0)
    want = np.where(counted, (m - z[np.arange(M), at]) + rest, 0.0)
    dz = 2 * U * d * (np.abs(ref["y"]) @ np.abs(W).T).max(1)
    x = 2 * dz + 2 * U * 88 + 2.0 ** -21 + 2 * U * (64 + V / 64)
    bound = np.where(counted, x * rest + 2 * U * want + np.where(z[np.arange(M), at] < m, 2 * dz, 0.0), 0.0)
    assert twins or want[counted].min() < 1e-6                           # what the test is about
    assert x.max() < 2e-3
    dhead = dict(h=dev_bf16(h_bits), gamma=dev(head["gamma"]), beta=dev(head["beta"]), W=dev_bf16(head["W"]))
    got = ee.ee_head_ce(dhead, dev(labels), 1e-5)
    err = np.abs(got["ce"].cpu().numpy().astype(np.float64) - want)
    worst = int(np.argmax(err - bound))
    assert (err <= bound).all(), (worst, err[worst], bound[worst], want[worst])
    dlse = dz + x + 2 * U * np.abs(ref["lse"])
    assert (np.abs(got["lse"].cpu().numpy().astype(np.float64) - ref["lse"]) <= dlse).all()
    mean = want.sum() / counted.sum()
    assert abs(float(got["loss"][0]) - mean) <= bound.max() + 2 * U * mean


@pytest.mark.parametrize("M,d,V", SIZES)
def test_the_gradient_of_nearly_certain_rows_keeps_its_digits(ee, M, d, V):
    """Row by row in dh.  The entries of G: e^(z - lse) is off by r = dz + dlse + 2^-21 of itself and rounded to bf16 (e = 2^-8); at the
    label e^(-ce) - 1 by what ce is off by, x (1 - p), plus 2 dz p where the label is not the largest logit, and 8u of itself; its
    rounding does not reach dy (test_gpu_ce_few_rows.py).  From G on as in test_gpu_ce.py."""
    h_bits, head, labels = _case(M, d, V, M + d + V)
    weights = np.ones(M, np.float32)
    ref = oracle.cross_entropy(h_bits, head, labels, weights)
    W, y, P = ref["W"], ref["y"], ref["P"]
    z = y @ W.T
    m, top = z.max(1), z.argmax(1)
    e = np.exp(z - m[:, None])
    e[np.arange(M), top] = 0.0
    ce = (m - z[np.arange(M), np.where(labels < 0, 0, labels)]) + np.log1p(e.sum(1))
    rows = np.flatnonzero(labels >= 0)
    at = labels[rows]
    G = ref["G"].copy()
    G[rows, at] = np.expm1(-ce[rows])                                    # 1 - p by its digits in 64 bits too
    dy = G @ W
    g, x_hat, s = head["gamma"].astype(np.float64), ref["xhat"], ref["rstd"]
    t = dy * g
    want = s * (t - t.mean(1, keepdims=True) - x_hat * (t * x_hat).mean(1, keepdims=True))
    dz = 2 * U * d * (np.abs(y) @ np.abs(W).T).max(1)
    x = 2 * dz + 2 * U * 88 + 2.0 ** -21 + 2 * U * (64 + V / 64)
    r = dz + (dz + x + 2 * U * np.abs(ref["lse"])) + 2.0 ** -21
    dG = np.where((labels >= 0)[:, None], r[:, None] * P * (1 + E) + E * np.abs(G), 0.0)
    off = np.abs(G[rows, at])
    dG[rows, at] = (x[rows] + 8 * U) * off + np.where(at != top[rows], 2 * dz[rows] * P[rows, at], 0.0)
    Ddy = dG @ np.abs(W) + 2 * U * (V + 40) * (np.abs(G) @ np.abs(W))
    ta, xa = np.abs(t), np.abs(x_hat)
    Dt = Ddy * g + 4 * U * ta
    inner = Dt + Dt.mean(1, keepdims=True) + xa * (Dt * xa).mean(1, keepdims=True)
    size = ta + ta.mean(1, keepdims=True) + xa * (ta * xa).mean(1, keepdims=True)
    bound = s * (inner + 2 * U * (d + 16) * size + 8 * U * (xa + 4.0) * (ta * (xa + 1)).mean(1, keepdims=True))
    bound = bound * (1 + E) + E * np.abs(want) + 1e-38
    dhead = dict(h=dev_bf16(h_bits), gamma=dev(head["gamma"]), beta=dev(head["beta"]), W=dev_bf16(head["W"]))
    fwd = ee.ee_head_ce(dhead, dev(labels), 1e-5)
    got = ee.ee_head_ce_grad(dhead, dev(labels), 1e-5, fwd, dce=dev(weights))
    err = np.abs(_np(got["dh"]) - want)
    worst = np.unravel_index(np.argmax(err / bound), err.shape)
    assert (err <= bound).all(), (worst, err[worst], bound[worst], want[worst], ce[worst[0]])
    # without the losses the same to what lse in fp32 allows
    rough = _np(ee.ee_head_ce_grad(dhead, dev(labels), 1e-5, {k: fwd[k] for k in ("lse", "loss")}, dce=dev(weights))["dh"])
    slack = 2 * U * np.abs(ref["lse"])[:, None] * s * (np.abs(W).max() * g).max() * (3 + xa)
    assert (np.abs(rough - want) <= bound + (1 + E) * (slack + 2 * dz[:, None] * s * (np.abs(W).max() * g).max() * (3 + xa))).all()


def test_losses_of_another_shape_are_refused(ee):
    h_bits, head, labels = _case(40, 64, 200, 1)
    dhead = dict(h=dev_bf16(h_bits), gamma=dev(head["gamma"]), beta=dev(head["beta"]), W=dev_bf16(head["W"]))
    fwd = ee.ee_head_ce(dhead, dev(labels), 1e-5)
    for bad in (fwd["ce"][:39], fwd["ce"].double(), fwd["ce"].cpu()):
        with pytest.raises(ValueError):
            ee.ee_head_ce_grad(dhead, dev(labels), 1e-5, dict(fwd, ce=bad))
