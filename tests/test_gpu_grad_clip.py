"""ee_grad_norm, ee_grad_clip and GradClip against fp64.

Bounds: the squares of eight (four in fp32) elements are added in fp32, at most 8 roundings of 2^-24 of the sum, everything above in fp64, and the root
halves a relative error: 2^-22 for the norm with its own rounding.  The factor has three more roundings and the product one, before the rounding
to the tensor's type (half a step: 2^-8, 2^-11, 2^-24)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _norm(grads):
    return math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))


def _check(ee, grads, max_norm, in_place):
    before = [g.clone() for g in grads]
    norm = _norm(before)
    out = None if in_place else [torch.full_like(g, 5.0) for g in grads]
    got = ee.ee_grad_clip(grads, max_norm, out=out)
    assert abs(got.item() - norm) <= 2.0 ** -22 * norm, (got.item(), norm)
    factor = min(1.0, max_norm / (norm + 1e-6))
    for g, b, o in zip(grads, before, grads if in_place else out):
        want = b.double() * factor
        half = HALF_STEP[g.dtype]
        lowest = float(torch.finfo(g.dtype).smallest_normal) * 2 * half
        assert ((o.double() - want).abs() <= (half * (1 + 2.0 ** -8) + 2.0 ** -21) * want.abs() + lowest).all()
        if factor == 1.0:
            assert torch.equal(o, b)
        if not in_place:
            assert torch.equal(g, b)


SETS = [[("bf16", 1)], [("f32", 3)], [("f16", 7), ("bf16", 0), ("f32", 1)], [("bf16", 16384)], [("bf16", 16385), ("f32", 8191)],
        [("f32", 100003), ("bf16", 4000001), ("f16", 20011)], [("bf16", 1000 + i) for i in range(17)], [("f32", 1 + i) for i in range(700)],
        [("bf16", 0)] * 3 + [("f32", 5)]]
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.mark.parametrize("which", range(len(SETS)))
@pytest.mark.parametrize("in_place", [True, False])
def test_norm_and_clip(ee, which, in_place):
    torch.manual_seed(which)
    grads = [(torch.randn(n, device="cuda") * 0.1).to(TYPES[t]) for t, n in SETS[which]]
    norm = _norm(grads)
    for max_norm in (norm * 0.3, norm * 2, 0.0):
        _check(ee, [g.clone() for g in grads], max_norm, in_place)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_unaligned_views_and_their_neighbours(ee, dtype):
    torch.manual_seed(3)
    for shift in (1, 3, 5):
        whole = torch.randn(40000, device="cuda").to(dtype)
        keep = whole.clone()
        view = whole[shift:shift + 33333]
        _check(ee, [view], 0.5, True)
        assert torch.equal(whole[:shift], keep[:shift]) and torch.equal(whole[shift + 33333:], keep[shift + 33333:])
        a, b = whole[:30000], torch.zeros(40000, device="cuda", dtype=dtype)[shift:shift + 30000]
        factor = 0.5 / (_norm([a]) + 1e-6)
        ee.ee_grad_clip([a], 0.5, out=[b])
        assert ((b.double() - a.double() * factor).abs() <= 2 * HALF_STEP[dtype] * a.double().abs() * factor + 1e-7).all()


@pytest.mark.parametrize("dtype,size", [(torch.float32, 1e30), (torch.float32, 1e-30), (torch.bfloat16, 1e30), (torch.bfloat16, 1e-35), (torch.float16, 6e-8)])
def test_magnitudes_whose_squares_leave_the_range(ee, dtype, size):
    g = (torch.randn(50001, device="cuda", dtype=torch.float64) * size).to(dtype)
    norm = _norm([g])
    assert norm > 0 and abs(ee.ee_grad_norm([g]).item() - norm) <= 2.0 ** -22 * norm
    h = torch.cat([g, torch.zeros(1000, device="cuda", dtype=dtype)])
    assert ee.ee_grad_norm([h]).item() == pytest.approx(norm, rel=2.0 ** -21)


def test_what_is_not_finite(ee):
    for bad in (float("nan"), float("inf")):
        g = torch.ones(100, device="cuda")
        g[40] = bad
        norm = ee.ee_grad_clip([g], 1.0)
        if math.isnan(bad):
            assert torch.isnan(norm).all() and torch.isnan(g).all()
        else:                                                            # 1 / inf = 0: zeros, and what was infinite is not a number
            assert torch.isinf(norm).all() and torch.isnan(g[40]) and not g[:40].any()


def test_halves_and_a_sum_in_between(ee):
    """What a program on several GPUs does: the norms of all are put together before the scaling."""
    grads = [torch.randn(5000, device="cuda"), torch.randn(333, device="cuda").bfloat16()]
    before = [g.clone() for g in grads]
    clip = ee.GradClip(grads)
    norm = clip.norm()
    norm.mul_(2.0)                                                       # as if three others had the same
    clip.scale(1.0)
    factor = 1.0 / (2 * _norm(before) + 1e-6)
    for g, b in zip(grads, before):
        assert ((g.double() - b.double() * factor).abs() <= 2 * HALF_STEP[g.dtype] * b.double().abs() * factor + 1e-9).all()


def test_the_same_bits_every_time_captured_and_on_two_streams(ee):
    torch.manual_seed(0)
    src = [torch.randn(n, device="cuda").to(t) for n, t in ((100003, torch.bfloat16), (77, torch.float32), (1 << 20, torch.float32))]
    want = [torch.empty_like(g) for g in src]
    norm = ee.ee_grad_clip(src, 1.0, out=want).clone()
    streams = [torch.cuda.Stream() for _ in range(2)]
    clips, graphs = [], []
    torch.cuda.synchronize()
    for s in streams:
        clip = ee.GradClip(src, out=[torch.empty_like(g) for g in src])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            clip(1.0)
            clip(1.0)
        clips.append(clip)
        graphs.append(g)
    for _ in range(5):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for clip in clips:
        assert torch.equal(clip.value, norm)
        for a, b in zip(clip.out, want):
            assert torch.equal(a, b)


def test_refusals(ee):
    g = torch.ones(10, device="cuda")
    for bad in ([g.double()], [g.cpu()], [torch.ones(4, 4, device="cuda").t()[:, :2]], [g, g], [g, None]):
        with pytest.raises(ValueError):
            ee.GradClip(bad)
    for bad in ([g], [g.bfloat16(), g], [g[:5], g]):
        with pytest.raises(ValueError):
            ee.GradClip([g, torch.ones(10, device="cuda")], out=bad)
    with pytest.raises(ee.EExitError):
        ee.ee_grad_clip([g], -1.0)
    with pytest.raises(ee.EExitError):
        ee.ee_grad_clip([g], float("nan"))
    with pytest.raises(ee.EExitError):
        ee.ee_grad_norm([g], workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    assert ee.ee_grad_norm([]).item() == 0 and ee.ee_grad_norm([g[:0]]).item() == 0
