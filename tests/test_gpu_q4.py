"""Heads held in 4 bits: packing bit for bit against the oracle, and the head against the oracle's head on the same weights."""
import numpy as np
import pytest
import torch

import gen
import oracle
from _util import ENTROPY_TOL, assert_head_matches, dev, dev_bf16, head_to_dev, oracle_head

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _bits(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


@pytest.mark.parametrize("V,d,group", [(1, 32, 32), (17, 96, 32), (40, 64, 64), (33, 192, 64), (130, 128, 128), (257, 384, 128), (1000, 1024, 64)])
def test_pack_and_unpack_are_exact(ee, V, d, group):
    rng = np.random.default_rng(V)
    W = rng.normal(0, 0.02, (V, d)).astype(np.float32)
    W[:: 3] *= np.exp(rng.normal(0, 8, W[:: 3].shape)).astype(np.float32)       # all magnitudes within a group
    W[V // 2, :group] = 0.0                                                      # a group of zeros: scale 0
    W[V // 3, 0] = 1e-38                                                         # next to the smallest normal numbers
    bits = gen.bf16_bits_from_f32(W)
    q4 = ee.ee_head_q4_pack(dev_bf16(bits), group)
    got = _bits(ee.ee_head_q4_unpack(q4))
    want = oracle.q4_values(bits, group)
    # -0 and 0 stand for the same value
    assert np.array_equal(np.where(got == 0x8000, 0, got), np.where(want == 0x8000, 0, want))
    again = ee.ee_head_q4_pack(dev_bf16(bits), group, out=q4)
    assert again is q4 and np.array_equal(_bits(ee.ee_head_q4_unpack(q4)), got)


def test_packing_ties_go_to_the_even_number(ee):
    w = np.zeros((3, 32), np.float32)
    w[0, :9] = [7.0, -7.0, 3.5, 2.5, 1.5, 0.5, -0.5, -2.5, 6.5]
    w[2] = w[0] * 2.0 ** -20
    got = oracle.bf16_decode(_bits(ee.ee_head_q4_unpack(ee.ee_head_q4_pack(dev_bf16(gen.bf16_bits_from_f32(w)), 32))))
    want = [7, -7, 4, 2, 2, 0, 0, -2, 6]
    assert list(got[0, :9]) == want and not got[1].any() and np.array_equal(got[2, :9], np.array(want) * 2.0 ** -20)


HEADS = [(1, 32, 1, 32), (1, 1024, 5000, 64), (2, 96, 47, 32), (7, 64, 16, 64), (8, 512, 50304, 32), (9, 128, 1000, 128), (16, 320, 515, 64),
         (17, 256, 3001, 32), (31, 384, 2049, 128), (33, 2560, 700, 128), (64, 1024, 2500, 64), (65, 64, 300, 64), (150, 192, 900, 32),
         (3, 8192, 200, 128), (40, 8192, 100, 64), (64, 4096, 90, 32)]


@pytest.mark.parametrize("M,d,V,group", HEADS)
def test_head_matches_the_oracle(ee, M, d, V, group):
    cfg = gen.make_config("c1", seed=17, planted=True, M=M, d=d, V=V, heads=1)
    head = cfg["heads"][0]
    hd, h = head_to_dev(head), dev_bf16(cfg["h"])
    q4 = ee.ee_head_q4_pack(hd["W"], group)
    W4 = oracle.q4_values(head["W"], group)
    tau = np.linspace(0.2, 3.0, M).astype(np.float32)
    for t in (1.0, tau):
        out = ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, q4, dev(t) if isinstance(t, np.ndarray) else t)
        assert_head_matches(out, oracle_head(cfg["h"], dict(head, W=W4), t), label=f"{M} {d} {V} {group}")
    again = ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, q4, dev(tau))
    for k in out:
        assert torch.equal(out[k], again[k]), k
    # the 16-bit head on what the packed weights stand for: the same logits up to the order of the sums, and to the elements of y (one
    # in 10^5) that are one bf16 step apart
    full = ee.ee_exit_head(h, hd["gamma"], hd["beta"], 1e-5, ee.ee_head_q4_unpack(q4), dev(tau))
    assert (full["entropy"] - out["entropy"]).abs().max().item() <= ENTROPY_TOL


def test_strides_ties_and_rows_behind_the_last(ee):
    M, d, V, group = 11, 128, 600, 64
    cfg = gen.make_config("c1", seed=3, planted=True, M=M, d=d, V=V, heads=1)
    hd = head_to_dev(cfg["heads"][0])
    h = dev_bf16(cfg["h"])
    q4 = ee.ee_head_q4_pack(hd["W"], group)
    want = ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, q4, 1.0)
    wide = torch.zeros((M, d + 40), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + d] = h
    out = {k: torch.full((M + 5,), 9, dtype=v.dtype, device="cuda") for k, v in want.items()}
    ee.ee_exit_head_q4(wide[:, 8:8 + d], hd["gamma"], hd["beta"], 1e-5, q4, 1.0, out=out)
    for k in want:
        assert torch.equal(out[k][:M], want[k]) and (out[k][M:] == 9).all(), k
    # equal rows of W: the lowest index wins
    W = hd["W"].clone()
    W[:] = W[5]
    tied = ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, ee.ee_head_q4_pack(W, group), 100.0)
    assert not tied["argmax"].any() and (tied["entropy"] - np.log(V)).abs().max().item() < 1e-5 and tied["exit_mask"].all()


def test_a_row_that_is_not_a_number_does_not_exit_and_leaves_the_others_alone(ee):
    M, d, V = 20, 64, 500
    cfg = gen.make_config("c1", seed=4, planted=True, M=M, d=d, V=V, heads=1)
    hd = head_to_dev(cfg["heads"][0])
    h = dev_bf16(cfg["h"])
    q4 = ee.ee_head_q4_pack(hd["W"], 32)
    want = ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, q4, 50.0)
    bad = h.clone()
    bad[3, 1], bad[18, 0] = float("nan"), float("inf")
    got = ee.ee_exit_head_q4(bad, hd["gamma"], hd["beta"], 1e-5, q4, 50.0)
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[3] = keep[18] = False
    for k in want:
        assert torch.equal(got[k][keep], want[k][keep]), k
    assert torch.isnan(got["entropy"][~keep]).all() and not got["exit_mask"][~keep].any() and want["exit_mask"].all()


def test_captured_and_on_two_streams(ee):
    M, d, V = 8, 512, 5000
    cfg = gen.make_config("c0", seed=5, planted=True, M=M, d=d, V=V)
    hd = head_to_dev(cfg["heads"][0])
    h = dev_bf16(cfg["h"])
    q4 = ee.ee_head_q4_pack(hd["W"], 64)
    want = {k: v.clone() for k, v in ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, q4, 1.0).items()}
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    calls, graphs = [], []
    for s in streams:
        with torch.cuda.stream(s):
            calls.append(ee.prepare_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, q4, 1.0, workspace=ee.new_exit_head_q4_workspace(M, q4)))
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


def test_refusals(ee):
    W = torch.zeros((40, 128), dtype=torch.bfloat16, device="cuda")
    h = torch.zeros((4, 128), dtype=torch.bfloat16, device="cuda")
    gamma = beta = torch.ones(128, device="cuda")
    for group in (16, 48, 256):
        with pytest.raises(ee.EExitError):
            ee.ee_head_q4_pack(W, group)
    with pytest.raises(ee.EExitError):
        ee.ee_head_q4_pack(torch.zeros((40, 96), dtype=torch.bfloat16, device="cuda"), 64)
    with pytest.raises(ValueError):
        ee.ee_head_q4_pack(W[:, :64], 64)                                # strided
    with pytest.raises(TypeError):
        ee.ee_head_q4_pack(W.float(), 64)
    q4 = ee.ee_head_q4_pack(W, 64)
    with pytest.raises(ValueError):
        ee.ee_head_q4_pack(W, 32, out=q4)                                # made for another group
    with pytest.raises(ValueError):
        ee.Q4Weights(q4.data[:100], 40, 128, 64)
    with pytest.raises(ValueError):
        ee.ee_exit_head_q4(h[:, :64], gamma, beta, 1e-5, q4, 1.0)        # another width
    with pytest.raises(ValueError):
        ee.ee_exit_head_q4(h, gamma[:64], beta, 1e-5, q4, 1.0)
    with pytest.raises(ValueError):
        ee.ee_exit_head_q4(h, gamma, beta, 1e-5, q4, torch.ones(3, device="cuda"))
    with pytest.raises(ValueError):
        ee.ee_exit_head_q4(h, gamma, beta, 1e-5, q4, 1.0, out=ee.new_outputs(3))
    with pytest.raises(ee.EExitError) as e:
        ee.ee_exit_head_q4(h, gamma, beta, 1e-5, q4, 1.0, workspace=torch.zeros(512, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 4
    empty = ee.ee_exit_head_q4(h[:0], gamma, beta, 1e-5, q4, 1.0)
    assert empty["argmax"].numel() == 0


@pytest.mark.parametrize("M,d", [(1, 96), (2, 2560), (3, 1056), (9, 1024), (16, 2048), (20, 1536)])
def test_rows_far_from_zero_need_their_squared_deviations(ee, M, d):
    """Half of the rows are 100 plus 0 or 1/2: mean of squares minus square of the mean keeps too few bits there, in some warps only."""
    rng = np.random.default_rng(d)
    cfg = gen.make_config("c1", seed=7, planted=True, M=M, d=d, V=333, heads=1)
    h = gen.f32_from_bf16_bits(cfg["h"])
    h[::2] = 100 + 0.5 * rng.integers(0, 2, h[::2].shape)
    bits = gen.bf16_bits_from_f32(h.astype(np.float32))
    head = cfg["heads"][0]
    hd = head_to_dev(head)
    out = ee.ee_exit_head_q4(dev_bf16(bits), hd["gamma"], hd["beta"], 1e-5, ee.ee_head_q4_pack(hd["W"], 32), 1.0)
    assert_head_matches(out, oracle_head(bits, dict(head, W=oracle.q4_values(head["W"], 32)), 1.0), label=f"{M} {d}")
