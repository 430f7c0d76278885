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


@pytest.mark.parametrize("half", [False, True])
def test_made_on_one_stream_and_called_on_another(ee, half):
    """The workspace is cleared on the stream where the object is made, here behind a tenth of a second of other work, in memory that held ones."""
    torch.manual_seed(0)
    grads = [torch.randn(n, device="cuda") for n in (100003, 77)]
    want = sum(float((g.double() ** 2).sum()) for g in grads) ** 0.5
    nbytes = ee.new_grad_norm_workspace(grads).numel()
    made, called = torch.cuda.Stream(), [torch.cuda.Stream() for _ in range(2)]
    out = [torch.empty_like(g) for g in grads]
    torch.cuda.synchronize()
    with torch.cuda.stream(made):
        ones = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
        del ones                                                         # the workspace is likely to get this memory
        torch.cuda._sleep(200_000_000)
        clip = ee.GradClip(grads, out=out)
    for s in called:
        with torch.cuda.stream(s):
            if half:
                clip.norm()
                clip.scale(1.0)
            else:
                clip(1.0)
        s.synchronize()
        assert made.query()                                              # what the call had to wait for
        assert abs(clip.value.item() - want) <= 2.0 ** -22 * want
        for g, o in zip(grads, out):
            assert ((o - g / want).abs() <= 1e-6 * g.abs() / want + 1e-30).all()
        clip.value.zero_()
        torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        clip(1.0)
    graph.replay()
    assert abs(clip.value.item() - want) <= 2.0 ** -22 * want
