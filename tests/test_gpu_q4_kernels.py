"""The two kernels behind ee_exit_head_q4 against each other's oracle, on sizes either may be given (EE_Q4_KERNEL forces one)."""
import numpy as np
import pytest
import torch

import gen
import oracle
from _util import assert_head_matches, dev, dev_bf16, head_to_dev, oracle_head

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


@pytest.mark.parametrize("kernel", ["stream", "gemm"])
@pytest.mark.parametrize("M,d,V,group", [(1, 32, 1, 32), (1, 64, 16, 64), (5, 96, 33, 32), (8, 512, 50304, 64), (16, 1024, 2369, 64), (17, 96, 5000, 32),
                                         (33, 640, 700, 128), (64, 64, 80000, 64), (65, 192, 2400, 32), (128, 256, 640, 128), (129, 64, 3000, 64),
                                         (3, 8192, 20, 128), (100, 2560, 300, 64), (20, 128, 152000, 128)])
def test_each_kernel_matches_the_oracle(ee, monkeypatch, kernel, M, d, V, group):
    monkeypatch.setenv("EE_Q4_KERNEL", kernel)
    cfg = gen.make_config("c1", seed=23, planted=True, M=M, d=d, V=V, heads=1)
    head = cfg["heads"][0]
    hd, h = head_to_dev(head), dev_bf16(cfg["h"])
    q4 = ee.ee_head_q4_pack(hd["W"], group)
    ws = ee.new_exit_head_q4_workspace(M, q4)
    tau = np.linspace(0.2, 3.0, M).astype(np.float32)
    out = ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, q4, dev(tau), workspace=ws)
    assert ee.ee_query_async_error(ws) == 0
    assert_head_matches(out, oracle_head(cfg["h"], dict(head, W=oracle.q4_values(head["W"], group)), tau), label=f"{kernel} {M} {d} {V} {group}")
    again = ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, q4, dev(tau), workspace=ws)
    for k in out:
        assert torch.equal(out[k], again[k]), k


@pytest.mark.parametrize("kernel", ["stream", "gemm"])
def test_not_a_number_stays_in_its_row(ee, monkeypatch, kernel):
    monkeypatch.setenv("EE_Q4_KERNEL", kernel)
    M, d, V = 40, 128, 900
    cfg = gen.make_config("c1", seed=4, planted=True, M=M, d=d, V=V, heads=1)
    hd, h = head_to_dev(cfg["heads"][0]), dev_bf16(cfg["h"])
    q4 = ee.ee_head_q4_pack(hd["W"], 32)
    want = ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, q4, 50.0)
    bad = h.clone()
    bad[7, 1], bad[39, 0] = float("nan"), float("-inf")
    got = ee.ee_exit_head_q4(bad, hd["gamma"], hd["beta"], 1e-5, q4, 50.0)
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[7] = keep[39] = False
    for k in want:
        assert torch.equal(got[k][keep], want[k][keep]), k
    assert torch.isnan(got["entropy"][~keep]).all() and not got["exit_mask"][~keep].any()


@pytest.mark.parametrize("kernel", ["stream", "gemm"])
@pytest.mark.parametrize("M,d,V,group", [(1, 32, 5, 32), (5, 96, 700, 32), (33, 640, 2500, 128), (100, 64, 60000, 64)])
def test_what_the_workspace_held_does_not_matter(ee, monkeypatch, kernel, M, d, V, group):
    monkeypatch.setenv("EE_Q4_KERNEL", kernel)
    cfg = gen.make_config("c1", seed=8, planted=True, M=M, d=d, V=V, heads=1)
    hd, h = head_to_dev(cfg["heads"][0]), dev_bf16(cfg["h"])
    q4 = ee.ee_head_q4_pack(hd["W"], group)
    ws = ee.new_exit_head_q4_workspace(M, q4)
    results = []
    for junk in (0, 255):
        ws[256:].fill_(junk)
        results.append({k: v.clone() for k, v in ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, q4, 1.0, workspace=ws).items()})
    for k in results[0]:
        assert torch.equal(results[0][k], results[1][k]), k
    assert torch.isfinite(results[1]["entropy"]).all()
