"""Heads in microscaled 4-bit floating point: what rows without a value give."""
import numpy as np
import pytest

import gen
from _util import dev_bf16, head_to_dev

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
