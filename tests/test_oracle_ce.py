"""Pins of the cross-entropy oracle: closed forms, and its gradient against central differences of its own loss."""
import math

import numpy as np

import gen
import oracle


def _f32(x):
    return gen.bf16_bits_from_f32(np.asarray(x, dtype=np.float32))


def test_closed_forms():
    # W = 0: every class equally likely, ce = ln V; gradient of W is (1/V - onehot) y / n
    M, d, V = 3, 8, 5
    rng = np.random.default_rng(0)
    head = dict(gamma=np.ones(d, np.float32), beta=np.zeros(d, np.float32), ln_eps=1e-5, W=_f32(np.zeros((V, d))))
    h = _f32(rng.normal(0, 1, (M, d)))
    labels = np.array([1, 4, 1])
    ref = oracle.cross_entropy(h, head, labels)
    assert np.allclose(ref["ce"], math.log(V), atol=1e-14) and abs(ref["loss"] - math.log(V)) < 1e-14 and ref["n"] == 3
    want = np.zeros((V, d))
    for i, lab in enumerate(labels):
        for v in range(V):
            want[v] += (1.0 / V - (v == lab)) * ref["y"][i] / 3.0
    assert np.allclose(ref["dW"], want, atol=1e-14)
    assert np.all(ref["dh"] == 0.0) and np.all(ref["dgamma"] == 0.0) and np.all(ref["dbeta"] == 0.0)
    # one class: certain, no gradient at all
    one = oracle.cross_entropy(h, dict(head, W=_f32(rng.normal(0, 1, (1, d)))), np.zeros(M, int))
    assert np.all(one["ce"] == 0.0) and np.all(one["dW"] == 0.0) and np.all(one["dh"] == 0.0)


def test_agrees_with_the_forward_oracle():
    cfg = gen.make_config("c1", seed=5, planted=True, M=20, d=64, V=300, heads=2)
    labels = np.random.default_rng(1).integers(0, 300, 20)
    kl = oracle.kl_to_teacher(cfg["h"], cfg["heads"][0], cfg["h"], cfg["heads"][1], labels=labels)
    ref = oracle.cross_entropy(cfg["h"], cfg["heads"][0], labels)
    assert np.allclose(ref["ce"], kl["ce"], atol=1e-12) and abs(ref["loss"] - kl["ce_loss"]) < 1e-12


def test_gradient_against_central_differences():
    M, d, V = 4, 16, 11
    rng = np.random.default_rng(3)
    gamma, beta = 1 + 0.2 * rng.normal(size=d), 0.1 * rng.normal(size=d)
    h, W = rng.normal(0.3, 1.5, (M, d)), rng.normal(0, 0.7, (V, d))
    labels = np.array([2, -1, 10, 2])
    weights = np.array([0.5, 3.0, -1.25, 0.75])

    def loss(h, gamma, beta, W):
        c = h - h.mean(1, keepdims=True)
        y = c / np.sqrt((c * c).mean(1, keepdims=True) + 1e-5) * gamma + beta
        z = y @ W.T
        return sum(w * (math.log(np.exp(z[i]).sum()) - z[i, lab]) for i, (lab, w) in enumerate(zip(labels, weights)) if lab >= 0)

    hb, Wb = _f32(h), _f32(W)
    head = dict(gamma=gamma.astype(np.float32), beta=beta.astype(np.float32), ln_eps=1e-5, W=Wb)
    at = [oracle.bf16_decode(hb), head["gamma"].astype(float), head["beta"].astype(float), oracle.bf16_decode(Wb)]
    ref = oracle.cross_entropy(hb, head, labels, weights, round_y=False)
    for k, name in enumerate(("dh", "dgamma", "dbeta", "dW")):
        x = at[k]
        for i in np.ndindex(x.shape):
            step = 1e-6
            up, down = [a.copy() for a in at], [a.copy() for a in at]
            up[k][i] += step
            down[k][i] -= step
            num = (loss(*up) - loss(*down)) / (2 * step)
            assert abs(num - ref[name][i]) < 1e-7 * (1 + abs(num)), (name, i, num, ref[name][i])
    assert np.all(ref["dh"][1] == 0.0)


def test_rows_that_are_not_counted():
    cfg = gen.make_config("c1", seed=6, planted=True, M=12, d=64, V=100, heads=1)
    head = cfg["heads"][0]
    labels = np.array([3, -1, 7, 100, 5, -100, 2, 2, 99, 0, 1 << 30, 50])
    ref = oracle.cross_entropy(cfg["h"], head, labels)
    keep = np.array([0, 2, 4, 6, 7, 8, 9, 11])
    part = oracle.cross_entropy(cfg["h"][keep], head, labels[keep])
    assert ref["n"] == 8 and abs(ref["loss"] - part["loss"]) < 1e-14
    assert np.allclose(ref["dW"], part["dW"], atol=1e-15) and np.allclose(ref["dh"][keep], part["dh"], atol=1e-15)
    none = oracle.cross_entropy(cfg["h"], head, np.full(12, -1))
    assert none["n"] == 0 and none["loss"] == 0.0 and not none["dW"].any() and not none["dh"].any()
