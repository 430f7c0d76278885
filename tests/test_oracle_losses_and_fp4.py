"""Pins of the oracles of the token losses and of 4-bit floating point: gradients against central differences, closed forms, and the formats
against torch's and against their definition by search."""
import numpy as np
import pytest
import torch

import oracle
from oracle.fp4 import ELEMENTS, quantise, round_e2m1, round_e4m3

V = 20


def _case(seed, M=40, S=6):
    rng = np.random.default_rng(seed)
    ce, old, ref = (np.abs(rng.normal(1, 0.7, M)) for _ in range(3))
    labels = rng.integers(-4, V, M)
    starts = np.concatenate([[0], np.sort(rng.integers(0, M + 1, S - 1)), [M]])
    return rng, ce, old, ref, labels, starts


def _differences(f, x, step=1e-6):
    g = np.zeros_like(x)
    for i in range(x.size):
        hi, lo = x.copy(), x.copy()
        hi[i] += step
        lo[i] -= step
        g[i] = (f(hi) - f(lo)) / (2 * step)
    return g


@pytest.mark.parametrize("by_sequence", [False, True])
def test_policy_gradient_against_differences(by_sequence):
    rng, ce, old, ref, labels, starts = _case(1)
    adv = rng.normal(0, 1, 6 if by_sequence else 40)
    args = dict(ref_ce=ref, kl_weight=0.3, clip=(0.2, 0.3), seq_start=starts if by_sequence else None)
    got = oracle.policy_loss(ce, old, adv, labels, V, **args)
    want = _differences(lambda c: oracle.policy_loss(c, old, adv, labels, V, **args)["loss"][0], ce)
    assert np.abs(got["dce"] - want).max() < 1e-8 and got["loss"][3] > 0 and not got["dce"][(labels < 0)].any()


def test_policy_loss_is_the_smaller_of_the_two_products():
    rng, ce, old, ref, labels, _ = _case(2)
    labels[:] = 1
    adv = rng.normal(0, 1, 40)
    r = np.exp(old - ce)
    want = -np.minimum(r * adv, np.clip(r, 0.8, 1.2) * adv)
    assert abs(oracle.policy_loss(ce, old, adv, labels, V)["loss"][1] - want.mean()) < 1e-14
    same = oracle.policy_loss(ce, ce, adv, labels, V, ref_ce=ce, kl_weight=1.0)
    assert abs(same["loss"][0] + adv.mean()) < 1e-14 and same["loss"][2] == 0 and np.abs(same["dce"] - adv / 40).max() < 1e-15


@pytest.mark.parametrize("with_ref,soft", [(True, 0.0), (False, 0.2)])
def test_preference_gradient_against_differences(with_ref, soft):
    _, ce, _, ref, labels, starts = _case(3)
    args = dict(ref_ce=ref if with_ref else None, beta=0.7, smoothing=soft)
    got = oracle.preference_loss(ce, labels, V, starts, **args)
    want = _differences(lambda c: oracle.preference_loss(c, labels, V, starts, **args)["loss"][0], ce)
    assert np.abs(got["dce"] - want).max() < 1e-8
    level = oracle.preference_loss(ce, labels, V, starts, ref_ce=ce, beta=0.7, smoothing=soft)
    assert np.abs(level["margin"]).max() == 0 and abs(level["loss"][0] - np.log(2)) < 1e-15


def test_formats():
    x = np.random.default_rng(0).normal(0, 3, 4000)
    x = np.concatenate([x, (ELEMENTS[1:] + ELEMENTS[:-1]) / 2, -(ELEMENTS[1:] + ELEMENTS[:-1]) / 2, [7.0, 100.0]])
    got = round_e2m1(x)
    dist = np.abs(np.abs(x)[:, None] - ELEMENTS)
    near = dist.min(1)
    assert np.array_equal(np.abs(np.abs(x) - np.abs(got)), near)
    ties = (dist == near[:, None]).sum(1) > 1
    assert ties.sum() == 14 and all(int(np.searchsorted(ELEMENTS, abs(v))) % 2 == 0 for v in got[ties])
    s = np.concatenate([np.exp(np.random.default_rng(1).uniform(-8, 5.8, 5000)), [2.0 ** -10, 3 * 2.0 ** -10, 1.0625, 1.1875, 340.0]]).astype(np.float32)
    want = torch.from_numpy(s).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(round_e4m3(s.astype(np.float64)), want)


@pytest.mark.parametrize("group", [16, 32])
def test_quantised_values_stay_near(group):
    x = np.random.default_rng(2).normal(0, 1, (8, 96)) * np.exp(np.random.default_rng(3).normal(0, 3, (8, 1)))
    x = torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    q, s = quantise(x, group, True)
    top = np.abs(x.reshape(8, -1, group)).max(2)
    v = q.reshape(8, -1, group) * s[:, :, None]
    # the widest step is 2 of 6 (or of 4, and up to 8 are cut to 6, with powers of two) around the top
    assert np.abs(v - x.reshape(v.shape)).max(2).max() <= (top * (0.26 if group == 32 else 0.23)).max()
    assert (np.abs(np.abs(v).max(2) - top) <= top * 0.26).all() and set(np.abs(q).ravel()) <= set(ELEMENTS)
