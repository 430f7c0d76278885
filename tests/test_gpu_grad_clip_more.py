"""GradClip: tensors that lie in one another, and streams."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def test_tensors_that_overlap_are_refused(ee):
    whole, other = torch.ones(100, device="cuda"), torch.ones(100, device="cuda")
    for bad in ([whole, whole], [whole, whole[50:]], [whole[10:20], whole], [whole[:60], other, whole[59:]], [whole[:50], whole[25:30].view(torch.bfloat16)]):
        with pytest.raises(ValueError, match="overlap"):
            ee.GradClip(bad)
    a, b = whole[:50], whole[50:]
    free = torch.ones(150, device="cuda")
    for out in ([b, a], [other[:50], other[25:75]], [other[:50], other[:50]], [free[:50], a], [a, whole[49:99]]):
        with pytest.raises(ValueError, match="overlap"):
            ee.GradClip([a, b], out=out)
    with pytest.raises(ValueError, match="overlap"):
        ee.GradClip([whole[:80]], out=[whole[20:]])
    # side by side, empty ones anywhere, and one of them in place
    ee.GradClip([a, b, whole[20:20], whole[:0]], out=[a, other[50:], whole[30:30], whole[:0]])(1.0)
    assert torch.equal(a, other[50:]) and (b == 1).all() and (a - 0.1).abs().max().item() < 1e-6
