"""ee_exit_head_q4 at widths where shared memory holds 8 rows of y and no more: both kernels, and which of them the call takes."""
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


@pytest.mark.parametrize("kernel", ["stream", "gemm", None])
@pytest.mark.parametrize("M,d,V,group", [(8, 8192, 700, 64), (9, 8192, 700, 32), (12, 8192, 2500, 128), (16, 6848, 400, 64), (16, 6784, 400, 64), (17, 7008, 333, 32)])
def test_more_rows_than_one_launch_of_the_streaming_kernel(ee, monkeypatch, kernel, M, d, V, group):
    if kernel:
        monkeypatch.setenv("EE_Q4_KERNEL", kernel)
    cfg = gen.make_config("c1", seed=29, planted=True, M=M, d=d, V=V, heads=1)
    head = cfg["heads"][0]
    hd, h = head_to_dev(head), dev_bf16(cfg["h"])
    tau = np.linspace(0.2, 3.0, M).astype(np.float32)
    out = ee.ee_exit_head_q4(h, hd["gamma"], hd["beta"], 1e-5, ee.ee_head_q4_pack(hd["W"], group), dev(tau))
    assert_head_matches(out, oracle_head(cfg["h"], dict(head, W=oracle.q4_values(head["W"], group)), tau), label=f"{kernel} {M} {d} {V} {group}")


@pytest.mark.parametrize("M,d,kernel", [(8, 8192, "stream"), (9, 8192, "gemm"), (16, 8192, "gemm"), (8, 6848, "stream"), (16, 6848, "gemm"),
                                        (16, 6784, "stream"), (17, 6784, "gemm")])
def test_a_batch_that_takes_two_passes_goes_to_the_other_kernel(ee, monkeypatch, M, d, kernel):
    """The kernels add up in different orders, so that of several rows' entropies some differ in their last bits."""
    V, group = 3000, 64
    rng = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randn(M, d, generator=rng, device="cuda").to(torch.bfloat16)
    q4 = ee.ee_head_q4_pack((0.02 * torch.randn(V, d, generator=rng, device="cuda")).to(torch.bfloat16), group)
    gamma, beta = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
    chosen = ee.ee_exit_head_q4(h, gamma, beta, 1e-5, q4, 2.0)["entropy"]
    for name in ("stream", "gemm"):
        monkeypatch.setenv("EE_Q4_KERNEL", name)
        same = torch.equal(ee.ee_exit_head_q4(h, gamma, beta, 1e-5, q4, 2.0)["entropy"], chosen)
        assert same == (name == kernel), name
