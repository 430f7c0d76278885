"""Heads in microscaled 4-bit floating point: what rows without a value give, and what the two head kernels do in runs of many tiles.  Bounds as in
test_gpu_fp4 (assert_close)."""
import numpy as np
import pytest
import torch

import gen
import oracle
from _util import dev_bf16, head_to_dev
from test_gpu_fp4 import assert_close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


@pytest.mark.parametrize("M", [5, 64, 65, 300])
def test_a_row_without_a_value_has_no_index_in_any_head(ee, M):
    d, V = 64, 500
    cfg = gen.make_config("c1", seed=4, planted=True, M=M, d=d, V=V, heads=1)
    hd = head_to_dev(cfg["heads"][0])
    bad = dev_bf16(cfg["h"]).clone()
    bad[3, 1], bad[4, 0] = float("nan"), float("inf")
    args = (bad, hd["gamma"], hd["beta"], 1e-5)
    outs = [ee.ee_exit_head_fp4(*args, ee.ee_head_fp4_pack(hd["W"], g), 50.0) for g in (16, 32)]
    outs += [ee.ee_exit_head_q4(*args, ee.ee_head_q4_pack(hd["W"], 32), 50.0), ee.ee_exit_head(*args, hd["W"], 50.0)]
    for out in outs:
        argmax = out["argmax"].cpu().numpy()
        assert (argmax[3:5] == 2 ** 31 - 1).all() and np.isnan(out["entropy"][3:5].cpu().numpy()).all() and not out["exit_mask"][3:5].any()
        assert (np.delete(argmax, [3, 4]) < V).all() and (argmax >= 0).all()


# What a CTA or a pair of them carries from tile to tile, on some 148 SMs.  Up to 64 rows: 313 to 469 weight tiles, two to four to a CTA, of one to four
# stages each, with the accumulators in turn.  Above: 5 to 21 tiles to a pair, of several units each; those of 1500 and 3000 rows cross from one row
# tile to the next.
LONG_RUNS = [(12, 256, 60000), (32, 640, 40000), (64, 1024, 50304), (203, 1056, 50257), (1000, 128, 50304), (3000, 1024, 5000), (3000, 2560, 5000), (1500, 2688, 6000)]


@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("M,d,V", LONG_RUNS)
def test_runs_of_many_tiles_match_the_oracle(ee, M, d, V, group):
    cfg = gen.make_config("c1", seed=23, planted=True, M=M, d=d, V=V, heads=1)
    head = cfg["heads"][0]
    hd = head_to_dev(head)
    fp4 = ee.ee_head_fp4_pack(hd["W"], group)
    workspace = ee.new_exit_head_fp4_workspace(M, fp4)
    out = ee.ee_exit_head_fp4(dev_bf16(cfg["h"]), hd["gamma"], hd["beta"], 1e-5, fp4, 1.0, workspace=workspace)
    assert_close(out, oracle.exit_head_fp4(cfg["h"], head, 1.0, group), d, V, f"{M} {d} {V} {group}")
    assert ee.ee_query_async_error(workspace) == 0


def test_packing_into_the_other_form_is_refused(ee):
    W = torch.zeros((128, 256), dtype=torch.bfloat16, device="cuda")
    whole, floating = ee.ee_head_q4_pack(W, 32), ee.ee_head_fp4_pack(W, 32)
    for pack, out in ((ee.ee_head_fp4_pack, whole), (ee.ee_head_q4_pack, floating)):
        with pytest.raises(TypeError):
            pack(W, 32, out=out)
    assert ee.ee_head_fp4_pack(W, 32, out=floating) is floating and ee.ee_head_q4_pack(W, 32, out=whole) is whole


def test_one_workspace_for_batches_of_all_sizes(ee):
    d, V = 256, 20000
    cfg = gen.make_config("c1", seed=6, planted=True, M=257, d=d, V=V, heads=1)
    hd, h = head_to_dev(cfg["heads"][0]), dev_bf16(cfg["h"])
    fp4 = ee.ee_head_fp4_pack(hd["W"], 16)
    workspace = ee.new_exit_head_fp4_workspace(257, fp4)
    for M in (257, 256, 1, 129, 64, 65, 9, 257):
        got = ee.ee_exit_head_fp4(h[:M], hd["gamma"], hd["beta"], 1e-5, fp4, 1.0, workspace=workspace)
        want = ee.ee_exit_head_fp4(h[:M], hd["gamma"], hd["beta"], 1e-5, fp4, 1.0)
        for k in want:
            assert torch.equal(got[k], want[k]), (M, k)


# Both forms of the activations' LayerNorm on both sides of the border between them, rows of all widths.
@pytest.mark.parametrize("M,d,V", [(2048, 640, 200), (2049, 640, 200), (2300, 1056, 130), (2100, 2592, 130), (2500, 8192, 100), (2049, 2560, 260)])
def test_activations_by_warps_and_by_ctas(ee, M, d, V):
    cfg = gen.make_config("c1", seed=29, planted=True, M=M, d=d, V=V, heads=1)
    head = cfg["heads"][0]
    hd = head_to_dev(head)
    for group in (16, 32):
        out = ee.ee_exit_head_fp4(dev_bf16(cfg["h"]), hd["gamma"], hd["beta"], 1e-5, ee.ee_head_fp4_pack(hd["W"], group), 1.0)
        assert_close(out, oracle.exit_head_fp4(cfg["h"], head, 1.0, group), d, V, f"{M} {d} {group}")


# Runs in which a pair keeps its row tile's activations: 128 tiles and more to a pair, of 13 to 20 units; short row tiles, so that every run goes through
# several, and long ones.  Rows are independent, so the oracle takes a sample of them.
@pytest.mark.parametrize("group", [16, 32])
@pytest.mark.parametrize("M,d,V", [(101200, 1664, 3000), (40000, 2048, 8000), (12300, 2560, 25200), (130000, 2528, 2400)])
def test_runs_that_keep_their_activations_match_the_oracle(ee, M, d, V, group):
    torch.manual_seed(M)
    W = (0.05 * torch.randn(V, d, device="cuda")).bfloat16()
    target = torch.randint(0, V, (M,), device="cuda")
    lean = torch.rand(M, 1, device="cuda") * 0.25
    h = (torch.randn(M, d, device="cuda") + lean * d ** 0.5 * torch.nn.functional.normalize(W[target].float(), dim=1)).bfloat16()
    gamma, beta = 1 + 0.1 * torch.randn(d, device="cuda"), 0.02 * torch.randn(d, device="cuda")
    fp4 = ee.ee_head_fp4_pack(W, group)
    workspace = ee.new_exit_head_fp4_workspace(M, fp4)
    out = ee.ee_exit_head_fp4(h, gamma, beta, 1e-5, fp4, 2.0, workspace=workspace)
    assert ee.ee_query_async_error(workspace) == 0
    rows = np.unique(np.concatenate([np.arange(20), np.arange(120, 136), np.arange(250, 262), np.arange(M - 20, M), np.random.default_rng(1).integers(0, M, 60)]))
    at = torch.from_numpy(rows).cuda()
    bits = lambda t: t.view(torch.int16).cpu().numpy().view(np.uint16)  # noqa: E731
    head = dict(gamma=gamma.cpu().numpy(), beta=beta.cpu().numpy(), W=bits(W), ln_eps=1e-5)
    assert_close({k: v[at] for k, v in out.items()}, oracle.exit_head_fp4(bits(h[at]), head, 2.0, group), d, V, f"{M} {d} {V} {group}")
    again = ee.ee_exit_head_fp4(h, gamma, beta, 1e-5, fp4, 2.0, workspace=workspace)
    for k in out:
        assert torch.equal(out[k], again[k]), k
