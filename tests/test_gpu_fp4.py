"""Heads in microscaled 4-bit floating point: packing bit for bit against the oracle, and the head against the oracle's."""
import numpy as np
import pytest
import torch

import gen
import oracle
from _util import GAP_MIN, MARGIN_MIN, dev, dev_bf16, head_to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _values(t):
    return t.float().cpu().numpy().astype(np.float64)


def assert_close(out, ref, d, V, label=""):
    """Entropy and largest probability to what fp32 sums give.  A logit is a sum of d products, 64 to a step: each step's rounding or cutting is
    at most 2^-22 of the magnitudes summed, which off by dz moves the entropy by at most 2 H dz and a probability by 2 p dz; the softmax's
    sums over V terms and the functions add 2^-18 of themselves."""
    got = {k: v.cpu().numpy() for k, v in out.items()}
    dz = (d / 64 + 4) * 2.0 ** -22 * ref["size"]
    H, p = ref["entropy"], ref["maxprob"]
    dH, dP = np.abs(got["entropy"] - H), np.abs(got["maxprob"] - p)
    tol_H, tol_P = 2 * H * dz + 2.0 ** -18 * H + 1e-30, (2 * dz + 2.0 ** -18) * p
    assert (dH <= tol_H).all(), f"{label}: entropy off by {dH.max():.2e}, {(dH / tol_H).max():.2f} of what it may"
    assert (dP <= tol_P).all(), f"{label}: largest probability {(dP / tol_P).max():.2f} of what it may"
    sure = ref["top2_gap"] >= GAP_MIN
    assert (got["argmax"] == ref["argmax"])[sure].all(), label
    sure = ref["tau_margin"] >= MARGIN_MIN
    assert (got["exit_mask"] == ref["exit_mask"])[sure].all(), label


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("V,d", [(1, 32), (17, 96), (129, 160), (33, 192), (257, 384), (1000, 1024), (5, 8192)])
def test_pack_and_unpack_are_exact(ee, V, d, group):
    rng = np.random.default_rng(V + group)
    W = rng.normal(0, 0.02, (V, d)).astype(np.float32)
    W[:: 3] *= np.exp(rng.normal(0, 6, W[:: 3].shape)).astype(np.float32)       # all magnitudes within a group
    W[V // 2, :group] = 0.0                                                      # a group of zeros
    W[V // 3, group - 1] = 1e-38                                                 # next to the smallest normal numbers
    bits = gen.bf16_bits_from_f32(W)
    fp4 = ee.ee_head_fp4_pack(dev_bf16(bits), group)
    got = _values(ee.ee_head_fp4_unpack(fp4))
    want = oracle.fp4_values(bits, group)
    bad = np.argwhere(got != want)
    assert bad.size == 0, bad[:5]
    again = ee.ee_head_fp4_pack(dev_bf16(bits), group, out=fp4)
    assert again is fp4 and np.array_equal(_values(ee.ee_head_fp4_unpack(fp4)), want)


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("scale", [2.0 ** -130, 2.0 ** -60, 1.0, 2.0 ** 120])
def test_ties_and_the_ends_of_the_range(ee, group, scale):
    w = np.zeros((2, 64), np.float32)
    w[0, :group] = np.resize([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -2.5, -5.0, 5.125, 4.875, 0.0, 7.0], group)
    w[1, group:2 * group] = np.resize([0.5, 0.001, 0.02, -0.3], group)
    bits = gen.bf16_bits_from_f32(w * np.float32(scale))
    got = _values(ee.ee_head_fp4_unpack(ee.ee_head_fp4_pack(dev_bf16(bits), group)))
    # at 2^-130 the values have more bits than bf16 has left (its grid ends at 2^-133): unpacking rounds them to it
    bad = np.argwhere(got != oracle.bf16_rne(oracle.fp4_values(bits, group)))
    assert bad.size == 0, bad[:5]
    zeros = ee.ee_head_fp4_unpack(ee.ee_head_fp4_pack(torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda"), group))
    assert not zeros.any()


HEADS = [(1, 32, 1), (1, 1024, 5000), (2, 96, 47), (7, 64, 16), (8, 512, 50304), (9, 128, 1000), (16, 320, 515), (17, 256, 3001), (31, 384, 2049),
         (33, 2560, 700), (64, 1024, 2500), (65, 64, 300), (100, 160, 900), (128, 512, 1111), (129, 512, 1111), (150, 192, 129), (300, 1056, 2000),
         (1100, 96, 700), (3, 8192, 200), (40, 8192, 100), (140, 8192, 90), (1030, 2592, 130),
         (20000, 96, 300), (40000, 32, 100), (12000, 2592, 260)]          # runs of tiles that go through several row tiles


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("M,d,V", HEADS)
def test_head_matches_the_oracle(ee, M, d, V, group):
    cfg = gen.make_config("c1", seed=17, planted=True, M=M, d=d, V=V, heads=1)
    head = cfg["heads"][0]
    hd, h = head_to_dev(head), dev_bf16(cfg["h"])
    fp4 = ee.ee_head_fp4_pack(hd["W"], group)
    tau = np.linspace(0.2, 3.0, M).astype(np.float32)
    workspace = ee.new_exit_head_fp4_workspace(M, fp4)
    for t in (1.0, tau):
        out = ee.ee_exit_head_fp4(h, hd["gamma"], hd["beta"], 1e-5, fp4, dev(t) if isinstance(t, np.ndarray) else t, workspace=workspace)
        assert_close(out, oracle.exit_head_fp4(cfg["h"], head, t, group), d, V, f"{M} {d} {V} {group}")
    again = ee.ee_exit_head_fp4(h, hd["gamma"], hd["beta"], 1e-5, fp4, dev(tau), workspace=workspace)
    for k in out:
        assert torch.equal(out[k], again[k]), k
    assert ee.ee_query_async_error(workspace) == 0


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("M", [11, 200])
def test_strides_ties_and_rows_behind_the_last(ee, M, group):
    d, V = 160, 600
    cfg = gen.make_config("c1", seed=3, planted=True, M=M, d=d, V=V, heads=1)
    hd = head_to_dev(cfg["heads"][0])
    h = dev_bf16(cfg["h"])
    fp4 = ee.ee_head_fp4_pack(hd["W"], group)
    want = ee.ee_exit_head_fp4(h, hd["gamma"], hd["beta"], 1e-5, fp4, 1.0)
    wide = torch.zeros((M, d + 40), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + d] = h
    out = {k: torch.full((M + 5,), 9, dtype=v.dtype, device="cuda") for k, v in want.items()}
    ee.ee_exit_head_fp4(wide[:, 8:8 + d], hd["gamma"], hd["beta"], 1e-5, fp4, 1.0, out=out)
    for k in want:
        assert torch.equal(out[k][:M], want[k]) and (out[k][M:] == 9).all(), k
    # equal rows of W: the lowest index wins
    W = hd["W"].clone()
    W[:] = W[5]
    tied = ee.ee_exit_head_fp4(h, hd["gamma"], hd["beta"], 1e-5, ee.ee_head_fp4_pack(W, group), 100.0)
    assert not tied["argmax"].any() and (tied["entropy"] - np.log(V)).abs().max().item() < 1e-5 and tied["exit_mask"].all()


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("M", [20, 300])
def test_a_row_that_is_not_a_number_does_not_exit_and_leaves_the_others_alone(ee, M, group):
    d, V = 64, 500
    cfg = gen.make_config("c1", seed=4, planted=True, M=M, d=d, V=V, heads=1)
    hd = head_to_dev(cfg["heads"][0])
    h = dev_bf16(cfg["h"])
    fp4 = ee.ee_head_fp4_pack(hd["W"], group)
    want = ee.ee_exit_head_fp4(h, hd["gamma"], hd["beta"], 1e-5, fp4, 50.0)
    bad = h.clone()
    bad[3, 1], bad[18, 0] = float("nan"), float("inf")
    got = ee.ee_exit_head_fp4(bad, hd["gamma"], hd["beta"], 1e-5, fp4, 50.0)
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[3] = keep[18] = False
    for k in want:
        assert torch.equal(got[k][keep], want[k][keep]), k
    assert torch.isnan(got["entropy"][~keep]).all() and not got["exit_mask"][~keep].any() and want["exit_mask"].all()


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("M", [5, 40, 150])
def test_scales_far_from_one_and_rows_far_from_zero(ee, M, group):
    """gamma of all magnitudes, rows of zeros after the LayerNorm, and rows of 100 plus 0 or 1/2."""
    d, V = 320, 333
    rng = np.random.default_rng(d + M)
    cfg = gen.make_config("c1", seed=7, planted=True, M=M, d=d, V=V, heads=1)
    head = dict(cfg["heads"][0])
    head["gamma"] = (np.exp(rng.normal(0, 4, d)) * 2.0 ** -20).astype(np.float32)
    head["beta"] = np.zeros(d, np.float32)
    head["W"] = gen.bf16_bits_from_f32(gen.f32_from_bf16_bits(head["W"]) * np.float32(2.0 ** 20))
    h = gen.f32_from_bf16_bits(cfg["h"])
    h[::2] = 100 + 0.5 * rng.integers(0, 2, h[::2].shape)
    h[1] = 3.0
    bits = gen.bf16_bits_from_f32(h.astype(np.float32))
    hd = head_to_dev(head)
    out = ee.ee_exit_head_fp4(dev_bf16(bits), hd["gamma"], hd["beta"], 1e-5, ee.ee_head_fp4_pack(hd["W"], group), 1.0)
    assert_close(out, oracle.exit_head_fp4(bits, dict(head, ln_eps=1e-5), 1.0, group), d, V)


@pytest.mark.parametrize("M", [8, 260])
def test_captured_and_on_two_streams(ee, M):
    d, V = 512, 5000
    cfg = gen.make_config("c0", seed=5, planted=True, M=M, d=d, V=V)
    hd = head_to_dev(cfg["heads"][0])
    h = dev_bf16(cfg["h"])
    fp4 = ee.ee_head_fp4_pack(hd["W"], 16)
    want = {k: v.clone() for k, v in ee.ee_exit_head_fp4(h, hd["gamma"], hd["beta"], 1e-5, fp4, 1.0).items()}
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    calls, graphs = [], []
    for s in streams:
        with torch.cuda.stream(s):
            calls.append(ee.prepare_exit_head_fp4(h, hd["gamma"], hd["beta"], 1e-5, fp4, 1.0, workspace=ee.new_exit_head_fp4_workspace(M, fp4)))
            calls[-1]()
    torch.cuda.synchronize()
    for s, call in zip(streams, calls):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
            call()
        graphs.append(g)
    for c in calls:
        for k in c.out:
            c.out[k].zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for c in calls:
        for k in want:
            assert torch.equal(c.out[k], want[k]), k


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("M", [4, 300])
def test_the_weights_are_data_of_the_stream(ee, M, group):
    """Packed again right before every call, the calls one behind the other in one graph: each answers from its own weights."""
    d, V = 256, 20000
    rng = np.random.default_rng(M)
    h = dev_bf16(gen.bf16_bits_from_f32(rng.normal(0, 1, (M, d)).astype(np.float32)))
    gamma, beta = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
    W = [dev_bf16(gen.bf16_bits_from_f32(rng.normal(0, 0.1, (V, d)).astype(np.float32))) for _ in range(3)]
    want = [ee.ee_exit_head_fp4(h, gamma, beta, 1e-5, ee.ee_head_fp4_pack(w, group), 5.0) for w in W]
    fp4 = ee.ee_head_fp4_pack(W[0], group)
    workspace = ee.new_exit_head_fp4_workspace(M, fp4)
    outs = [ee.new_outputs(M) for _ in W]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for w, out in zip(W, outs):
            ee.ee_head_fp4_pack(w, group, out=fp4)
            ee.ee_exit_head_fp4(h, gamma, beta, 1e-5, fp4, 5.0, out=out, workspace=workspace)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, outs):
        for k in a:
            assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("M", [1, 5, 17, 130])
def test_entropies_of_nearly_certain_rows_keep_their_digits(ee, M):
    """Entropies down to 1e-6 and below, to the same part of themselves (assert_close)."""
    d, V, group = 64, 200, 16
    rng = np.random.default_rng(12)
    w_bits = gen.bf16_bits_from_f32(rng.normal(0, 0.3, (V, d)).astype(np.float32))
    h = oracle.fp4_values(w_bits, group)[rng.integers(0, V, M)] * 3 + rng.normal(0, 0.1, (M, d))
    h_bits = gen.bf16_bits_from_f32(h.astype(np.float32))
    head = dict(gamma=np.full(d, 1.2, np.float32), beta=np.zeros(d, np.float32), W=w_bits, ln_eps=1e-5)
    y4 = oracle.exit_head_fp4(h_bits, head, 0.5, group)
    z = _logits(h_bits, head, group)
    dz = z - z.max(1, keepdims=True)
    e = np.exp(dz)
    rest = np.sort(e, axis=1)[:, :-1].sum(1)                             # without the largest term
    y4["entropy"], y4["maxprob"] = np.log1p(rest) - (e * dz).sum(1) / (1.0 + rest), 1.0 / (1.0 + rest)
    got = ee.ee_exit_head_fp4(dev_bf16(h_bits), dev(head["gamma"]), dev(head["beta"]), 1e-5, ee.ee_head_fp4_pack(dev_bf16(w_bits), group), 0.5)
    assert y4["entropy"].min() < 1e-3                                    # what the test is about
    assert_close(got, y4, d, V)


def _logits(h_bits, head, group):
    from oracle.ce_loss import _rows, bf16_by_f32
    from oracle.fp4 import values
    return values(bf16_by_f32(_rows(h_bits, head)[2]), group, True) @ oracle.fp4_values(head["W"], group).T


def test_refusals(ee):
    W = torch.zeros((40, 128), dtype=torch.bfloat16, device="cuda")
    h = torch.zeros((4, 128), dtype=torch.bfloat16, device="cuda")
    gamma = beta = torch.ones(128, device="cuda")
    for group in (8, 48, 64):
        with pytest.raises(ee.EExitError):
            ee.ee_head_fp4_pack(W, group)
    with pytest.raises(ee.EExitError):
        ee.ee_head_fp4_pack(torch.zeros((40, 72), dtype=torch.bfloat16, device="cuda"), 16)
    with pytest.raises(ValueError):
        ee.ee_head_fp4_pack(W[:, :64], 16)                               # strided
    with pytest.raises(TypeError):
        ee.ee_head_fp4_pack(W.float(), 16)
    fp4 = ee.ee_head_fp4_pack(W, 16)
    with pytest.raises(ValueError):
        ee.ee_head_fp4_pack(W, 32, out=fp4)                              # made for another group
    with pytest.raises(ValueError):
        ee.Fp4Weights(fp4.data[:100], 40, 128, 16)
    with pytest.raises(ValueError):
        ee.ee_exit_head_fp4(h[:, :64], gamma, beta, 1e-5, fp4, 1.0)      # another width
    with pytest.raises(ValueError):
        ee.ee_exit_head_fp4(h, gamma[:64], beta, 1e-5, fp4, 1.0)
    with pytest.raises(ValueError):
        ee.ee_exit_head_fp4(h, gamma, beta, 1e-5, fp4, torch.ones(3, device="cuda"))
    with pytest.raises(ValueError):
        ee.ee_exit_head_fp4(h, gamma, beta, 1e-5, fp4, 1.0, out=ee.new_outputs(3))
    with pytest.raises(ee.EExitError) as e:
        ee.ee_exit_head_fp4(h, gamma, beta, 1e-5, fp4, 1.0, workspace=torch.zeros(512, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 4
    assert ee.ee_exit_head_fp4(h[:0], gamma, beta, 1e-5, fp4, 1.0)["argmax"].numel() == 0
