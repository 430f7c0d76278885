"""ee_head_ce and ee_head_ce_grad against the fp64 oracle.

Bounds, element by element (u = 2^-24, e = 2^-8, the largest relative error of one rounding to bf16):
  z      products of bf16 numbers are exact in fp32; d additions, each off by at most 2u of the running magnitude:
         dz = 2 u d sum_j |w_j y_j|, taken at its largest over a row
  lse    dz, plus the relative error of the sum of exponentials: 2^-21 for an exponential (the approximate instruction's
         2^-22 and its argument's rounding for logits below 64 in magnitude) and 2u for each of at most 64 + V / 64
         additions or rescalings, plus 2u |lse|; ce adds another dz and 2u |ce|
  G      relative error of P: r = dz + dlse + 2^-21; then one rounding to bf16:  dG = |w| P r (1 + e) + e |G|
  dW     sum_i dG |y| + 2u M sum_i |G| |y| + e |dW| (+ e more of the first part for the product of roundings)
  dy     sum_v dG |W| + 2u (V + pieces) sum_v |G| |W|, and through the LayerNorm with 2u d for its sums
The bounds are sums of magnitudes, so results sit well inside them; a wrong term does not.
"""
import numpy as np
import pytest
import torch

import gen
import oracle
from _util import dev, dev_bf16, head_to_dev

pytestmark = pytest.mark.gpu
U, E = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def bounds(ref, gamma):
    y, W, G, P, w = ref["y"], ref["W"], ref["G"], ref["P"], np.abs(ref["weights"])
    M, d = y.shape
    V = W.shape[0]
    dz = 2 * U * d * (np.abs(y) @ np.abs(W).T).max(axis=1) if M else np.zeros(0)
    dlse = dz + 2.0 ** -21 + 2 * U * (64 + V / 64) + 2 * U * np.abs(ref["lse"])
    dce = dlse + dz + 2 * U * np.abs(ref["ce"])
    r = dz + dlse + 2.0 ** -21
    dG = (w * r)[:, None] * P * (1 + E) + E * np.abs(G) * (1 + U * 8)
    aG = np.abs(G)
    dW = dG.T @ np.abs(y) + 2 * U * (M + 2) * (aG.T @ np.abs(y))
    dW = dW * (1 + E) + E * np.abs(ref["dW"]) + 1e-38
    Ddy = dG @ np.abs(W) + 2 * U * (V + 40) * (aG @ np.abs(W))
    g, x, s = np.abs(gamma).astype(np.float64), np.abs(ref["xhat"]), ref["rstd"]
    t = np.abs(ref["dy"]) * g
    Dt = Ddy * g + 4 * U * t
    inner = Dt + Dt.mean(1, keepdims=True) + x * (Dt * x).mean(1, keepdims=True)
    size = t + t.mean(1, keepdims=True) + x * (t * x).mean(1, keepdims=True)
    h_mag = x + 4.0                              # (h - mean) / sigma is off by u times |mean| / sigma too: inputs keep that below 4
    dh = s * (inner + 2 * U * (d + 16) * size + 8 * U * h_mag * (t * (x + 1)).mean(1, keepdims=True))
    dh = dh * (1 + E) + E * np.abs(ref["dh"]) + 1e-38
    adds = 2 * U * (M + 16)
    dgamma = ((Ddy * x).sum(0) + adds * (np.abs(ref["dy"]) * (x + 4.0)).sum(0)) * (1 + E) + E * np.abs(ref["dgamma"]) + 1e-38
    dbeta = (Ddy.sum(0) + adds * np.abs(ref["dy"]).sum(0)) * (1 + E) + E * np.abs(ref["dbeta"]) + 1e-38
    return dict(lse=dlse, ce=dce, dW=dW, dh=dh, dgamma=dgamma, dbeta=dbeta, loss=dce.max() if M else 0.0)


def make(M, d, V, planted=True, seed=31, ignored=0.25):
    cfg = gen.make_config("c1", seed=seed, planted=planted, M=M, d=d, V=V, heads=1)
    rng = np.random.default_rng(M + d + V)
    labels = rng.integers(0, V, size=M)
    if planted:                                   # half the labels are the token the row follows
        tok = gen.make_planting(seed, f"c1/planted/d{d}/V{V}", d, V)["tokens"][cfg["j"]]
        labels = np.where(rng.random(M) < 0.5, tok, labels)
    labels[rng.random(M) < ignored] = -1
    labels[0] = V - 1                             # the last column of the ragged last tile
    return cfg, labels.astype(np.int32)


def device_head(cfg):
    hd = head_to_dev(cfg["heads"][0])
    return dict(h=dev_bf16(cfg["h"]), gamma=hd["gamma"], beta=hd["beta"], W=hd["W"])


def check(got, ref, bnd, names, label=""):
    for name in names:
        err = np.abs(_np(got[name]) - ref[name])
        worst = np.unravel_index(np.argmax(err / bnd[name]), err.shape)
        assert np.all(err <= bnd[name]), (label, name, worst, err[worst], bnd[name][worst], ref[name][worst])


GRADS = ("dW", "dh", "dgamma", "dbeta")
SIZES = [(1, 8, 1), (1, 64, 257), (3, 72, 65), (64, 128, 400), (128, 8, 300), (129, 320, 515), (257, 136, 1000), (300, 64, 2049),
         (700, 72, 700), (1000, 520, 3001), (40, 8192, 130), (2, 256, 20011)]


@pytest.mark.parametrize("M,d,V", SIZES)
@pytest.mark.parametrize("planted", [False, True])
def test_loss_and_gradient_match_the_oracle(ee, M, d, V, planted):
    cfg, labels = make(M, d, V, planted)
    head, lab = device_head(cfg), dev(labels)
    ref = oracle.cross_entropy(cfg["h"], cfg["heads"][0], labels)
    bnd = bounds(ref, cfg["heads"][0]["gamma"])
    fwd = ee.ee_head_ce(head, lab, 1e-5)
    check(fwd, ref, bnd, ("lse", "ce"))
    assert abs(float(fwd["loss"][0]) - ref["loss"]) <= bnd["loss"] and float(fwd["loss"][1]) == ref["n"]
    out = ee.ee_head_ce_grad(head, lab, 1e-5, fwd)
    check(out, ref, bnd, GRADS)
    again = ee.ee_head_ce_grad(head, lab, 1e-5, ee.ee_head_ce(head, lab, 1e-5))
    for k in GRADS:
        assert torch.equal(out[k], again[k]), k                          # fixed orders throughout


def test_pieces_of_the_vocabulary(ee):
    """More logits than one piece of the gradient holds: dy is added up over the pieces, dW comes piece by piece."""
    M, d, V = 2100, 64, 50304
    cfg, labels = make(M, d, V)
    labels[:6] = [0, 255, 256, 25087, 25088, V - 1]
    head, lab = device_head(cfg), dev(labels)
    ref = oracle.cross_entropy(cfg["h"], cfg["heads"][0], labels)
    bnd = bounds(ref, cfg["heads"][0]["gamma"])
    fwd = ee.ee_head_ce(head, lab, 1e-5)
    check(fwd, ref, bnd, ("lse", "ce"))
    check(ee.ee_head_ce_grad(head, lab, 1e-5, fwd), ref, bnd, GRADS)


def test_row_weights_and_incoming_gradient(ee):
    M, d, V = 150, 64, 700
    cfg, labels = make(M, d, V)
    head, lab = device_head(cfg), dev(labels)
    w = np.random.default_rng(2).normal(0, 1, M).astype(np.float32)
    w[5] = 0.0
    ref = oracle.cross_entropy(cfg["h"], cfg["heads"][0], labels, w)
    fwd = ee.ee_head_ce(head, lab, 1e-5)
    got = ee.ee_head_ce_grad(head, lab, 1e-5, fwd, dce=dev(w))
    check(got, ref, bounds(ref, cfg["heads"][0]["gamma"]), GRADS)
    assert not got["dh"][5].any()
    up = 0.37
    ref = oracle.cross_entropy(cfg["h"], cfg["heads"][0], labels, np.full(M, np.float64(np.float32(up)) / max(1, int((labels >= 0).sum()))))
    got = ee.ee_head_ce_grad(head, lab, 1e-5, fwd, dloss=torch.tensor([up], device="cuda"))
    check(got, ref, bounds(ref, cfg["heads"][0]["gamma"]), GRADS)


def test_rows_that_are_not_counted_may_hold_anything(ee):
    M, d, V = 140, 72, 500
    cfg, labels = make(M, d, V, ignored=0.4)
    labels[:4] = [-1, V, -2 ** 31, 2 ** 31 - 1]
    labels[139] = -1
    clean = device_head(cfg)
    dirty = dict(clean, h=clean["h"].clone())
    lab = dev(labels)
    off = torch.from_numpy(np.flatnonzero((labels < 0) | (labels >= V))).cuda()
    dirty["h"][off[0]] = float("nan")
    dirty["h"][off[1]] = float("inf")
    dirty["h"][off[2:], 3] = -float("inf")
    f0, f1 = ee.ee_head_ce(clean, lab, 1e-5), ee.ee_head_ce(dirty, lab, 1e-5)
    assert torch.equal(f0["ce"], f1["ce"]) and torch.equal(f0["loss"], f1["loss"]) and not f1["ce"][off].any()
    for dce in (None, torch.ones(M, device="cuda")):
        g0, g1 = ee.ee_head_ce_grad(clean, lab, 1e-5, f0, dce=dce), ee.ee_head_ce_grad(dirty, lab, 1e-5, f1, dce=dce)
        for k in GRADS:
            assert torch.equal(g0[k], g1[k]), k
        assert not g1["dh"][off].any()
    # a counted row that is NaN shows in the loss
    bad = dict(clean, h=clean["h"].clone())
    on = int(np.flatnonzero((labels >= 0) & (labels < V))[3])
    bad["h"][on, 1] = float("nan")
    f = ee.ee_head_ce(bad, lab, 1e-5)
    assert torch.isnan(f["ce"][on]) and torch.isnan(f["loss"][0])
    # none counted: nothing but zeros
    none = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    f = ee.ee_head_ce(dirty, none, 1e-5)
    assert not f["loss"].any() and not f["ce"].any()
    g = ee.ee_head_ce_grad(dirty, none, 1e-5, f)
    for k in GRADS:
        assert not g[k].any(), k


def test_strides_partial_outputs_and_accumulation(ee):
    M, d, V = 130, 136, 300
    cfg, labels = make(M, d, V)
    head, lab = device_head(cfg), dev(labels)
    fwd = ee.ee_head_ce(head, lab, 1e-5)
    full = ee.ee_head_ce_grad(head, lab, 1e-5, fwd)
    wide = torch.full((M, d + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :d] = head["h"]
    strided = dict(head, h=wide[:, :d])
    dh_wide = torch.full((M + 2, d + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    out = ee.ee_head_ce_grad(strided, lab, 1e-5, ee.ee_head_ce(strided, lab, 1e-5), out=dict(dh=dh_wide[1:M + 1, :d]))
    assert torch.equal(out["dh"], full["dh"])
    assert (dh_wide[0] == 5).all() and (dh_wide[M + 1] == 5).all() and (dh_wide[:, d:] == 5).all()
    only = ee.ee_head_ce_grad(head, lab, 1e-5, fwd, out=dict(dW=torch.empty_like(full["dW"])))
    assert torch.equal(only["dW"], full["dW"])
    only = ee.ee_head_ce_grad(head, lab, 1e-5, fwd, out=dict(dgamma=torch.empty_like(full["dgamma"]), dbeta=torch.empty_like(full["dbeta"])))
    assert torch.equal(only["dgamma"], full["dgamma"]) and torch.equal(only["dbeta"], full["dbeta"])
    # accumulation: the fp32 gradient plus the old value, rounded once
    rng = np.random.default_rng(9)
    old = {k: dev_bf16(gen.bf16_bits_from_f32(rng.normal(0, 1e-3, full[k].shape).astype(np.float32))) for k in ("dW", "dgamma", "dbeta")}
    got = ee.ee_head_ce_grad(head, lab, 1e-5, fwd, accumulate=True, out=dict({k: v.clone() for k, v in old.items()}, dh=torch.empty_like(full["dh"])))
    ref = oracle.cross_entropy(cfg["h"], cfg["heads"][0], labels)
    bnd = bounds(ref, cfg["heads"][0]["gamma"])
    assert torch.equal(got["dh"], full["dh"])
    for k in old:
        want = ref[k] + _np(old[k])
        assert np.all(np.abs(_np(got[k]) - want) <= bnd[k] + E * np.abs(want)), k


def test_a_captured_step_replays_on_another_stream_beside_an_eager_one(ee):
    M, d, V = 200, 64, 900
    cfg, labels = make(M, d, V)
    head, lab = device_head(cfg), dev(labels)
    want_f = {k: v.clone() for k, v in ee.ee_head_ce(head, lab, 1e-5).items()}
    want = {k: v.clone() for k, v in ee.ee_head_ce_grad(head, lab, 1e-5, want_f).items()}
    ws, ws2 = ee.new_head_ce_grad_workspace(M, d, V), ee.new_head_ce_grad_workspace(M, d, V)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fwd = ee.ee_head_ce(head, lab, 1e-5, workspace=ws)
        out = ee.ee_head_ce_grad(head, lab, 1e-5, fwd, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ee.ee_head_ce(head, lab, 1e-5, out=fwd, workspace=ws)
        ee.ee_head_ce_grad(head, lab, 1e-5, fwd, out=out, workspace=ws)
    for k in out:
        out[k].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.replay()
        graph.replay()
    f2 = ee.ee_head_ce(head, lab, 1e-5, workspace=ws2)                   # meanwhile, with a workspace of its own
    g2 = ee.ee_head_ce_grad(head, lab, 1e-5, f2, workspace=ws2)
    torch.cuda.synchronize()
    for k in GRADS:
        assert torch.equal(out[k], want[k]) and torch.equal(g2[k], want[k]), k
    assert ee.ee_query_async_error(ws) == 0 and ee.ee_query_async_error(ws2) == 0


@pytest.mark.parametrize("M,d,V", [(1, 8, 1), (64, 72, 300), (130, 64, 900), (648, 128, 13018), (1000, 64, 13018), (500, 1216, 3546), (2100, 8, 40000)])
def test_what_the_workspace_held_does_not_matter(ee, M, d, V):
    """13018 = 73 tiles of 176 columns and 170 more, 38 short of a whole block of 64: every column that the products read is written."""
    cfg, labels = make(M, d, V)
    head, lab = device_head(cfg), dev(labels)
    ws = ee.new_head_ce_grad_workspace(M, d, V)
    results = []
    for junk in (0.0, float("nan")):
        ws[256:256 + (ws.numel() - 256) // 4 * 4].view(torch.float32).fill_(junk)
        fwd = ee.ee_head_ce(head, lab, 1e-5, workspace=ws)
        ws[256:256 + (ws.numel() - 256) // 4 * 4].view(torch.float32).fill_(junk)
        results.append(dict(fwd, **ee.ee_head_ce_grad(head, lab, 1e-5, fwd, workspace=ws)))
    for k in results[0]:
        assert torch.isfinite(results[1][k].float()).all() and torch.equal(results[0][k], results[1][k]), k


def test_no_rows(ee):
    head = dict(h=torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), gamma=torch.ones(64, device="cuda"),
                beta=torch.zeros(64, device="cuda"), W=torch.ones((50, 64), dtype=torch.bfloat16, device="cuda"))
    lab = torch.empty(0, dtype=torch.int32, device="cuda")
    f = ee.ee_head_ce(head, lab, 1e-5)
    assert not f["loss"].any()
    g = ee.ee_head_ce_grad(head, lab, 1e-5, f)
    assert not g["dW"].any() and not g["dgamma"].any() and not g["dbeta"].any() and g["dh"].shape == (0, 64)


def test_refusals(ee):
    cfg, labels = make(6, 64, 90)
    head, lab = device_head(cfg), dev(labels)
    fwd = ee.ee_head_ce(head, lab, 1e-5)
    with pytest.raises(ValueError):
        ee.ee_head_ce(head, lab.long(), 1e-5)                            # 64-bit labels
    with pytest.raises(ValueError):
        ee.ee_head_ce(head, lab[:5], 1e-5)                               # too few
    with pytest.raises(ValueError):
        ee.ee_head_ce(dict(head, W=head["W"][:, :32]), lab, 1e-5)        # another width
    with pytest.raises(ValueError):
        ee.ee_head_ce_grad(head, lab, 1e-5, fwd, dce=torch.ones(5, device="cuda"))
    with pytest.raises(ValueError):
        ee.ee_head_ce_grad(head, lab, 1e-5, fwd, accumulate=True)        # nothing to add to
    with pytest.raises(ValueError):
        ee.ee_head_ce_grad(head, lab, 1e-5, fwd, out=dict(dW=torch.empty((90, 64), device="cuda")))      # fp32
    with pytest.raises(ValueError):
        ee.ee_head_ce_grad(head, lab, 1e-5, dict(fwd, lse=fwd["lse"][:4]))
    with pytest.raises(ee.EExitError) as e:                              # row weights and the mean's gradient together
        ee.ee_head_ce_grad(head, lab, 1e-5, fwd, dce=torch.ones(6, device="cuda"), dloss=torch.ones(1, device="cuda"))
    assert e.value.code == 2
    with pytest.raises(ee.EExitError) as e:                              # dgamma without dbeta
        ee.ee_head_ce_grad(head, lab, 1e-5, fwd, out=dict(dgamma=torch.empty(64, dtype=torch.bfloat16, device="cuda")))
    assert e.value.code == 1
    with pytest.raises(ee.EExitError) as e:                              # the forward call's workspace is too small for the gradient
        ee.ee_head_ce_grad(head, lab, 1e-5, fwd, workspace=ee.new_head_ce_workspace(6, 64, 90))
    assert e.value.code == 4
    with pytest.raises(ee.EExitError) as e:                              # row stride not a multiple of eight
        ee.ee_head_ce(dict(head, h=torch.empty((6, 68), dtype=torch.bfloat16, device="cuda")[:, :64]), lab, 1e-5)
    assert e.value.code == 2
