"""Values at which a formula of the token losses read literally would be 0 times infinity.  Bounds as in test_gpu_token_loss: the exponentials' arguments
are rounded once, 2^-24 of at most 16, everything else adds a few 2^-24, together 2^-19 of the magnitudes."""
import numpy as np
import pytest
import torch

import oracle
from _util import dev

pytestmark = pytest.mark.gpu
R = 2.0 ** -19


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _np(t):
    return t.cpu().numpy().astype(np.float64)


def _forward(ce, labels, V):
    return {"ce": dev(ce), "loss": dev(np.array([0.0, ((labels >= 0) & (labels < V)).sum()], np.float32))}


@pytest.mark.parametrize("gap", [np.inf, -np.inf, 100.0])
def test_a_divergence_without_bound_is_infinite(ee, gap):
    """exp(g) - 1 - g of an infinite g, on either side, and where the exponential leaves fp32."""
    V, ce, labels = 10, np.full(6, 2.0, np.float32), np.array([0, 1, -1, 2, 3, 4], np.int32)
    ref = ce.copy()
    ref[3] = ce[3] - np.float32(gap)
    got = ee.ee_policy_loss(_forward(ce, labels, V), dev(labels), V, dev(ce), dev(np.ones(6, np.float32)), ref_ce=dev(ref), kl_weight=0.1)
    loss = _np(got["loss"])
    assert loss[0] == np.inf and abs(loss[1] + 1.0) <= R and loss[2] == np.inf and loss[3] == 0
    others = _np(got["dce"])[[0, 1, 4, 5]]
    assert np.abs(others - 0.2).max() <= R and _np(got["dce"])[2] == 0 and not np.isnan(_np(got["dce"])).any()


@pytest.mark.parametrize("by_sequence", [False, True])
@pytest.mark.parametrize("gap", [88.0, 100.0, np.inf])
def test_a_penalty_of_weight_zero_only_watches(ee, by_sequence, gap):
    """One counted token far from the reference: the divergence is reported, the loss and the weights do not know of it."""
    rng = np.random.default_rng(0)
    M, V = 300, 50
    ce = np.abs(rng.normal(0, 1.5, M)).astype(np.float32)
    old, ref = (np.abs(ce + rng.normal(0, s, M)).astype(np.float32) for s in (0.3, 0.5))
    labels = rng.integers(0, V, M).astype(np.int32)
    labels[::3] = -1
    ref[4] = ce[4] - np.float32(gap)
    starts = np.array([0, 100, 300], np.int32) if by_sequence else None
    adv = rng.normal(0, 1, 2 if by_sequence else M).astype(np.float32)
    args = dict(seq_start=None if starts is None else dev(starts))
    got = ee.ee_policy_loss(_forward(ce, labels, V), dev(labels), V, dev(old), dev(adv), ref_ce=dev(ref), kl_weight=0.0, **args)
    without = ee.ee_policy_loss(_forward(ce, labels, V), dev(labels), V, dev(old), dev(adv), **args)
    want = oracle.policy_loss(ce, old, adv, labels, V, None, 0.0, (0.2, 0.2), starts)
    assert torch.equal(got["dce"], without["dce"]) and torch.equal(got["loss"][[0, 1, 3]], without["loss"][[0, 1, 3]])
    size = np.abs(np.where(want["dce"] == 0, 1.0 / M, want["dce"]))
    assert (np.abs(_np(got["dce"]) - want["dce"]) <= R * size).all()
    assert abs(_np(got["loss"])[0] - want["loss"][0]) <= R * 4                # a mean of |adv| e^x, each below 4
    assert _np(got["loss"])[2] > 1e30


@pytest.mark.parametrize("by_sequence", [False, True])
def test_an_advantage_of_zero_asks_for_nothing(ee, by_sequence):
    """Also where the ratio of the probabilities leaves fp32, or the drafting head gave the token none; a cross-entropy that is not a number stays one."""
    V, labels = 10, np.zeros(6, np.int32)
    ce, old = np.zeros(6, np.float32), np.array([100.0, np.inf, 1.0, 100.0, 0.0, 0.05], np.float32)
    adv = np.array([0, -0.0, 0, 0, 1, -1], np.float32)
    starts = None
    if by_sequence:
        starts, adv = dev(np.array([0, 4, 6], np.int32)), np.array([0, 1], np.float32)
    got = ee.ee_policy_loss(_forward(ce, labels, V), dev(labels), V, dev(old), dev(adv), seq_start=starts)
    w = np.array([0.25] * 4 + [0.5] * 2) / 2 if by_sequence else np.full(6, 1 / 6)
    a = np.repeat(adv, [4, 2]) if by_sequence else adv
    want = w * a * np.exp(np.where(a == 0, 0.0, old))
    assert np.abs(_np(got["dce"]) - want).max() <= R and abs(_np(got["loss"])[0] + want.sum()) <= R and _np(got["loss"])[3] == 0
    ce[0] = np.nan
    got = ee.ee_policy_loss(_forward(ce, labels, V), dev(labels), V, dev(old), dev(adv), seq_start=starts)
    assert np.isnan(_np(got["dce"])[0]) and np.isnan(_np(got["loss"])[0]) and not np.isnan(_np(got["dce"])[1:]).any()


def test_sizes_beyond_32_bits_are_refused(ee):
    """2^32 + n tokens or labels' values are n to a 32-bit int, and the call answered for those."""
    small = torch.zeros(4, device="cuda")
    labels, starts = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    forward = {"ce": small, "loss": torch.ones(2, device="cuda")}
    for V in ((1 << 32) + 10, 10 - (1 << 32), 1 << 40):
        with pytest.raises(ee.EExitError):
            ee.ee_policy_loss(forward, labels, V, small, small)
        with pytest.raises(ee.EExitError):
            ee.ee_preference_loss(forward, labels, V, starts)
    many = torch.empty((1 << 32) + 5, device="cuda")
    forward, out = {"ce": many, "loss": torch.ones(2, device="cuda")}, {"loss": torch.zeros(4, device="cuda"), "margin": torch.zeros(1, device="cuda"), "dce": many}
    with pytest.raises(ee.EExitError):
        ee.ee_policy_loss(forward, many.view(torch.int32), 10, many, many, out=out)
    with pytest.raises(ee.EExitError):
        ee.ee_preference_loss(forward, many.view(torch.int32), 10, starts, out=out)


# What walks a unit: a warp, a CTA, a cluster of eight or of sixteen, units of ordinary and of very unequal lengths.
@pytest.mark.parametrize("M,S", [(140001, 2), (300001, 25), (20000, 100), (30000, 600), (30000, 300), (200000, 1), (60000, 7), (1000003, 148)])
@pytest.mark.parametrize("skewed", [False, True])
def test_policy_loss_whatever_walks_a_sequence(ee, M, S, skewed):
    rng = np.random.default_rng(M + S)
    V, ce, old, ref, labels, starts = _batch(rng, M, S, skewed)
    adv = rng.normal(0, 1, S).astype(np.float32)
    want = oracle.policy_loss(ce, old, adv, labels, V, ref, 0.1, (0.2, 0.2), starts)
    workspace = ee.new_token_loss_workspace()
    args = (_forward(ce, labels, V), dev(labels), V, dev(old), dev(adv))
    got = [ee.ee_policy_loss(*args, ref_ce=dev(ref), kl_weight=0.1, seq_start=dev(starts), workspace=workspace) for _ in range(2)]
    n = np.maximum(np.add.reduceat(np.append(labels >= 0, False), starts[:-1]) * (starts[1:] > starts[:-1]), 1)
    size = np.repeat(np.abs(adv) * 5 + 0.5, np.diff(starts)) / (np.repeat(n, np.diff(starts)) * S)      # |a| e^x + the penalty's part, x below 1.6
    assert (np.abs(_np(got[0]["dce"]) - want["dce"]) <= R * size).all()
    assert np.abs(_np(got[0]["loss"]) - want["loss"]).max() <= R * 5 * (1 + np.abs(adv).mean())
    assert torch.equal(got[0]["dce"], got[1]["dce"]) and torch.equal(got[0]["loss"], got[1]["loss"])


@pytest.mark.parametrize("M,P", [(140001, 2), (130001, 12), (400001, 30), (50000, 40), (30000, 600), (60000, 600), (200000, 1), (2000003, 148)])
@pytest.mark.parametrize("skewed", [False, True])
def test_preference_loss_whatever_walks_a_pair(ee, M, P, skewed):
    rng = np.random.default_rng(M + P)
    V, ce, _, ref, labels, starts = _batch(rng, M, 2 * P, skewed)
    want = oracle.preference_loss(ce, labels, V, starts, ref, 0.1, 0.1)
    workspace = ee.new_token_loss_workspace()
    args = (_forward(ce, labels, V), dev(labels), V, dev(starts))
    got = [ee.ee_preference_loss(*args, ref_ce=dev(ref), smoothing=0.1, workspace=workspace) for _ in range(2)]
    m = want["margin"]
    assert (np.abs(_np(got[0]["margin"]) - m) <= 2.0 ** -23 * np.abs(m) + 1e-9).all()
    assert (np.abs(_np(got[0]["dce"]) - want["dce"]) <= R * (1 + np.abs(m).max()) * np.abs(want["dce"]) + R * 0.1 * 0.1 / P).all()
    assert np.abs(_np(got[0]["loss"]) - want["loss"]).max() <= R * (1 + np.abs(want["loss"]).max() + np.abs(m).max())
    for k in got[0]:
        assert torch.equal(got[0][k], got[1][k]), k


def _batch(rng, M, n, skewed):
    """Tokens, a third of them not counted, and boundaries: nearly equal lengths, or one sequence of half of all tokens and some empty ones."""
    V = 100
    ce = np.abs(rng.normal(0, 1.5, M)).astype(np.float32)
    old, ref = (np.abs(ce + np.clip(rng.normal(0, 0.3, M), -0.8, 0.8)).astype(np.float32) for _ in range(2))
    labels = np.where(rng.random(M) < 0.3, -1, rng.integers(0, V, M)).astype(np.int32)
    starts = np.linspace(0, M, n + 1).astype(np.int32)
    if skewed and n > 1:
        starts = np.concatenate([[0], np.sort(rng.integers(M // 2, M + 1, n - 1)), [M]]).astype(np.int32)
        starts[-2] = starts[-1]
    return V, ce, old, ref, labels, starts


@pytest.mark.parametrize("long", [513, 2049, 30000])
def test_long_units_that_warps_leave_to_their_ctas(ee, long):
    """Several to a CTA, the last unit of all among them, of ordinary ones of 20 tokens."""
    rng = np.random.default_rng(long)
    lengths = np.full(1000, 20)
    lengths[[0, 3, 5, 6, 500, 999]] = long
    lengths[[4, 501]] = 0
    starts = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    V, ce, old, ref, labels, _ = _batch(rng, int(starts[-1]), 1, False)
    adv = rng.normal(0, 1, 1000).astype(np.float32)
    forward, lab, at = _forward(ce, labels, V), dev(labels), dev(starts)
    out = ee.ee_policy_loss(forward, lab, V, dev(old), dev(adv), ref_ce=dev(ref), kl_weight=0.1, seq_start=at)
    want = oracle.policy_loss(ce, old, adv, labels, V, ref, 0.1, (0.2, 0.2), starts)
    n = np.maximum([(labels[a:b] >= 0).sum() for a, b in zip(starts[:-1], starts[1:])], 1)
    size = np.repeat((np.abs(adv) * 5 + 0.5) / (n * 1000.0), lengths)
    assert (np.abs(_np(out["dce"]) - want["dce"]) <= R * size).all() and np.abs(_np(out["loss"]) - want["loss"]).max() <= R * 10
    out = ee.ee_preference_loss(forward, lab, V, at, ref_ce=dev(ref))
    want = oracle.preference_loss(ce, labels, V, starts, ref)
    m = want["margin"]
    assert (np.abs(_np(out["margin"]) - m) <= 2.0 ** -23 * np.abs(m) + 1e-9).all()
    assert (np.abs(_np(out["dce"]) - want["dce"]) <= R * (1 + np.abs(m).max()) * np.abs(want["dce"])).all()
    assert np.abs(_np(out["loss"]) - want["loss"]).max() <= R * (1 + np.abs(want["loss"]).max() + np.abs(m).max())
