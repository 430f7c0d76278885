"""ee_policy_loss and ee_preference_loss against the fp64 oracle.

Bounds (u = 2^-24): x = old_ce - ce and g = ce - ref_ce are taken in fp64 and rounded once, which moves their exponentials by u |x| and u |g| of
themselves; the functions are good to 2^-22, products and the weight's rounding add a few u.  Together, with |x|, |g| < 16: 2^-19 of the
magnitudes a value is made of.  Sums are fp64.  The margin is rounded once, the slope's exponential moved by u |m| of itself."""
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


def _tokens(rng, M, V, masked=0.3, junk=True):
    ce = np.abs(rng.normal(0, 1.5, M)).astype(np.float32)
    old = np.abs(ce + rng.normal(0, 0.3, M)).astype(np.float32)
    ref = np.abs(ce + rng.normal(0, 0.5, M)).astype(np.float32)
    old[: M // 8], ref[: M // 8] = ce[: M // 8], ce[: M // 8]            # a token that has not moved at all
    labels = rng.integers(0, V, M).astype(np.int32)
    labels[rng.random(M) < masked] = -1
    out = labels < 0
    labels[out] = rng.choice([-1, V, -2 ** 31, 2 ** 31 - 1], out.sum())
    if junk:
        for x in (ce, old, ref):
            x[out] = rng.choice([np.nan, np.inf, -np.inf, 3e38], out.sum())
    return ce, old, ref, labels


def _starts(rng, M, n, gap=0):
    """n + 1 boundaries of ragged sequences, empty ones among them; `gap` rows before the first and behind the last."""
    inner = np.sort(rng.integers(gap, max(M - gap, gap) + 1, n + 1))
    if n > 3:
        inner[2] = inner[1]
    if gap == 0:
        inner[0], inner[-1] = 0, M
    return inner.astype(np.int32)


def _forward(ee, ce, labels, V):
    n = ((labels >= 0) & (labels < V)).sum()
    return {"ce": dev(ce), "loss": dev(np.array([0.0, n], np.float32))}


def _check_policy(got, ref, args, kl_weight, label):
    dce = _np(got["dce"])
    size = np.abs(ref["dce"]) + args["scale"]
    bad = np.abs(dce - ref["dce"]) > R * size
    assert not bad.any(), (label, np.flatnonzero(bad)[:5], dce[bad][:5], ref["dce"][bad][:5])
    assert (np.abs(_np(got["loss"]) - ref["loss"]) <= R * args["loss_scale"] + 1e-30).all(), (label, got["loss"], ref["loss"])


def _policy_scales(ce, old, ref, adv, labels, V, kl_weight, starts):
    """Sums of magnitudes behind a token's weight and behind the means."""
    M = ce.size
    counted = (labels >= 0) & (labels < V)
    scale, total = np.zeros(M), np.zeros(4)
    units = [(0, M)] if starts is None else list(zip(starts[:-1], starts[1:]))
    for u, (a, b) in enumerate(units):
        at = np.flatnonzero(counted[a:b]) + a
        if at.size == 0:
            continue
        w = 1.0 / (at.size * len(units))
        x, g = old[at].astype(np.float64) - ce[at], (ce[at].astype(np.float64) - ref[at] if ref is not None else np.zeros(at.size))
        A = np.abs(adv[at] if starts is None else np.full(at.size, adv[u])).astype(np.float64)
        # |e^g - 1| is as good as its own size; the series of e^g - 1 - g too
        kl, e = np.abs(np.expm1(g) - g) * 2, np.abs(np.expm1(g)) * 4
        scale[at] = w * (A * np.exp(x) + kl_weight * e)
        pol = A * np.maximum(np.exp(x), 1.3)
        total += w * np.array([(pol + kl_weight * kl).sum(), pol.sum(), kl.sum(), at.size])
    return dict(scale=scale, loss_scale=total)


@pytest.mark.parametrize("M", [1, 2, 31, 257, 5000, 300001])
@pytest.mark.parametrize("kl_weight", [None, 0.0, 0.04])
def test_policy_loss_over_tokens(ee, M, kl_weight):
    rng = np.random.default_rng(M)
    V = 1000
    ce, old, ref, labels = _tokens(rng, M, V)
    adv = rng.normal(0, 1, M).astype(np.float32)
    adv[::7] = 0.0
    r = None if kl_weight is None else ref
    kw = kl_weight or 0.0
    want = oracle.policy_loss(ce, old, adv, labels, V, r, kw, (0.2, 0.28))
    got = ee.ee_policy_loss(_forward(ee, ce, labels, V), dev(labels), V, dev(old), dev(adv), ref_ce=None if r is None else dev(r), kl_weight=kw,
                            clip=(0.2, 0.28))
    _check_policy(got, want, _policy_scales(ce, old, r, adv, labels, V, kw, None), kw, M)


@pytest.mark.parametrize("M,S,gap", [(1, 1, 0), (1, 5, 0), (40, 3, 0), (3000, 3000, 0), (5000, 700, 9), (5000, 3, 100), (70000, 2, 0), (70000, 30, 0), (70000, 90, 1),
                                     (300001, 9000, 0)])
def test_policy_loss_over_sequences(ee, M, S, gap):
    rng = np.random.default_rng(M + S)
    V = 77
    ce, old, ref, labels = _tokens(rng, M, V)
    starts = _starts(rng, M, S, gap)
    if S > 2:
        labels[starts[1]:starts[2] + 3] = -1                             # sequences without a counted token
    adv = rng.normal(0, 1, S).astype(np.float32)
    want = oracle.policy_loss(ce, old, adv, labels, V, ref, 0.1, (0.1, 0.3), starts)
    workspace = ee.new_token_loss_workspace()
    out = ee.new_policy_loss_outputs(M)
    out["dce"].fill_(float("nan"))
    got = ee.ee_policy_loss(_forward(ee, ce, labels, V), dev(labels), V, dev(old), dev(adv), ref_ce=dev(ref), kl_weight=0.1, clip=(0.1, 0.3),
                            seq_start=dev(starts), out=out, workspace=workspace)
    _check_policy(got, want, _policy_scales(ce, old, ref, adv, labels, V, 0.1, starts), 0.1, (M, S))
    again = ee.ee_policy_loss(_forward(ee, ce, labels, V), dev(labels), V, dev(old), dev(adv), ref_ce=dev(ref), kl_weight=0.1, clip=(0.1, 0.3),
                              seq_start=dev(starts), workspace=workspace)
    assert torch.equal(got["dce"], again["dce"]) and torch.equal(got["loss"], again["loss"])


def test_policy_loss_at_its_borders(ee):
    """Ratios exactly at, one step inside and one step outside the clip; nothing counted; a probability of zero when drafted."""
    V = 10
    high = np.float32(np.log1p(0.2))
    ce = np.zeros(6, np.float32)
    old = np.array([np.nextafter(high, np.float32(0)), np.nextafter(high, np.float32(1)), np.float32(np.log1p(-0.2)) * np.float32(1.0001), -0.1, 40.0, 0.0], np.float32)
    adv = np.array([1, 1, -1, -1, 2, 0], np.float32)
    labels = np.zeros(6, np.int32)
    want = oracle.policy_loss(ce, old, adv, labels, V)
    got = ee.ee_policy_loss(_forward(ee, ce, labels, V), dev(labels), V, dev(old), dev(adv))
    assert np.array_equal(_np(got["dce"]) == 0, want["dce"] == 0) and abs(_np(got["loss"])[3] - want["loss"][3]) < 1e-7
    none = np.full(6, -1, np.int32)
    for starts in (None, np.array([0, 2, 2, 6], np.int32)):
        a = adv if starts is None else adv[:3]
        got = ee.ee_policy_loss(_forward(ee, ce, none, V), dev(none), V, dev(old), dev(a), seq_start=None if starts is None else dev(starts))
        assert not got["dce"].any() and not got["loss"].any()
    empty = ee.ee_policy_loss(_forward(ee, ce[:0], none[:0], V), dev(none[:0]), V, dev(old[:0]), dev(adv[:0]))
    assert not empty["loss"].any()


@pytest.mark.parametrize("M,P,gap", [(0, 2, 0), (1, 1, 0), (50, 4, 0), (4001, 8, 0), (5000, 900, 3), (20000, 40, 0), (70000, 1, 50), (300001, 3, 0), (300001, 100, 0), (300001, 3000, 0)])
@pytest.mark.parametrize("with_ref,smoothing", [(True, 0.0), (False, 0.1)])
def test_preference_loss(ee, M, P, gap, with_ref, smoothing):
    rng = np.random.default_rng(M + P)
    V = 500
    ce, _, ref, labels = _tokens(rng, M, V)
    starts = _starts(rng, M, 2 * P, gap)
    beta = 0.1 if with_ref else 0.01
    want = oracle.preference_loss(ce, labels, V, starts, ref if with_ref else None, beta, smoothing)
    out = ee.new_preference_loss_outputs(M, P)
    out["dce"].fill_(float("nan"))
    got = ee.ee_preference_loss(_forward(ee, ce, labels, V), dev(labels), V, dev(starts), ref_ce=dev(ref) if with_ref else None, beta=beta,
                                smoothing=smoothing, out=out)
    m = want["margin"]
    assert (np.abs(_np(got["margin"]) - m) <= 2.0 ** -23 * np.abs(m) + 1e-9).all()
    assert np.abs(_np(got["loss"]) - want["loss"]).max() <= R * (1 + np.abs(want["loss"]).max() + np.abs(m).max())
    # (where e^-|m| leaves fp32's normal numbers, it and the weight are rounded to its grid of 2^-149)
    size = R * (1 + np.abs(m).max()) * np.abs(want["dce"]) + (R * smoothing * beta / P) + 2.0 ** -148
    assert (np.abs(_np(got["dce"]) - want["dce"]) <= size).all()
    counted = (labels >= 0) & (labels < V)
    assert not _np(got["dce"])[~counted].any()


def test_boundaries_out_of_range_touch_nothing_outside(ee):
    """Boundaries are data: whatever they say, only the M rows are read and written."""
    M, V = 100, 10
    ce, old, ref, labels = _tokens(np.random.default_rng(0), M, V, junk=False)
    starts = np.array([-5, 40, 20, 2 ** 31 - 1, -2 ** 31], np.int32)
    whole = torch.full((M + 64,), 7.0, device="cuda")
    out = {"loss": torch.empty(4, device="cuda"), "dce": whole[32:32 + M]}
    ee.ee_policy_loss(_forward(ee, ce, labels, V), dev(labels), V, dev(old), dev(np.ones(4, np.float32)), seq_start=dev(starts), out=out)
    out["margin"] = torch.empty(2, device="cuda")
    ee.ee_preference_loss(_forward(ee, ce, labels, V), dev(labels), V, dev(starts), out=out)
    assert (whole[:32] == 7).all() and (whole[32 + M:] == 7).all() and not torch.isnan(whole).any()


def test_captured_and_on_two_streams(ee):
    rng = np.random.default_rng(1)
    M, S, V = 9000, 60, 50
    ce, old, ref, labels = _tokens(rng, M, V)
    f, lab, starts, adv = _forward(ee, ce, labels, V), dev(labels), dev(_starts(rng, M, S)), dev(rng.normal(0, 1, S).astype(np.float32))
    want = [ee.ee_policy_loss(f, lab, V, dev(old), adv, seq_start=starts), ee.ee_preference_loss(f, lab, V, starts, ref_ce=dev(ref))]
    old, ref = dev(old), dev(ref)
    torch.cuda.synchronize()
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    for s in streams:
        with torch.cuda.stream(s):
            workspace = ee.new_token_loss_workspace()
            calls = [ee.prepare_policy_loss(f, lab, V, old, adv, seq_start=starts, workspace=workspace),
                     ee.prepare_preference_loss(f, lab, V, starts, ref_ce=ref, workspace=workspace)]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            for c in calls:
                c()
                c()
        graphs.append(g)
        outs.append([c.out for c in calls])
    for _ in range(5):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for o in outs:
        for a, b in zip(o, want):
            for k in b:
                assert torch.equal(a[k], b[k]), k


def test_refusals(ee):
    M, V = 12, 10
    ce, labels, adv = torch.zeros(M, device="cuda"), torch.zeros(M, dtype=torch.int32, device="cuda"), torch.ones(M, device="cuda")
    f = {"ce": ce, "loss": torch.zeros(2, device="cuda")}
    starts = torch.tensor([0, 4, 12], dtype=torch.int32, device="cuda")
    for bad in (dict(old_ce=ce[:5]), dict(adv=adv[:5]), dict(labels=labels.long()), dict(seq_start=starts), dict(seq_start=starts[:1]),
                dict(ref_ce=ce.double()), dict(out={"loss": ce, "dce": ce}), dict(workspace=ce), dict(old_ce=torch.zeros(2 * M, device="cuda")[::2])):
        args = dict(old_ce=ce, adv=adv, labels=labels)
        args.update(bad)
        with pytest.raises(ValueError):
            ee.ee_policy_loss(f, args.pop("labels"), V, args.pop("old_ce"), args.pop("adv"), **args)
    for bad in (dict(clip=(-0.1, 0.2)), dict(clip=(1.5, 0.2)), dict(clip=(0.2, float("nan"))), dict(kl_weight=0.1), dict(kl_weight=-1.0, ref_ce=ce)):
        with pytest.raises(ee.EExitError):
            ee.ee_policy_loss(f, labels, V, ce, adv, **bad)
    with pytest.raises(ee.EExitError):
        ee.ee_policy_loss(f, labels, 0, ce, adv)
    for bad in (dict(seq_start=starts[:2]), dict(seq_start=None), dict(seq_start=starts.long()), dict(ref_ce=ce[:3])):
        with pytest.raises(ValueError):
            ee.ee_preference_loss(f, labels, V, **{"seq_start": starts, **bad})
    for bad in (dict(beta=-1.0), dict(smoothing=1.5), dict(smoothing=float("nan"))):
        with pytest.raises(ee.EExitError):
            ee.ee_preference_loss(f, labels, V, starts, **bad)
