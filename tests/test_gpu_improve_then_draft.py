"""The losses over tokens, the clipping and the 4-bit floating-point head as a program uses them, one after the other: a head's cross-entropies,
the loss of what it drafted, the gradient with those weights, its norm, the step, packing, and drafting with the result.

Bounds: ee_head_ce_grad's own (test_gpu_ce), for the weights that the loss call wrote; the clipped gradient is one more rounding to bf16 of a
product with a factor that is good to 2^-20."""
import numpy as np
import pytest
import torch

import gen
import oracle
from _util import dev, dev_bf16
from test_gpu_ce import bounds, check
from test_gpu_fp4 import assert_close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _bits(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Head:
    """A head and one step of improving it, in buffers of its own."""

    def __init__(self, ee, M, d, V, kind, seed=3):
        self.ee, self.M, self.d, self.V, self.kind = ee, M, d, V, kind
        rng = np.random.default_rng(seed)
        self.W = dev_bf16(gen.bf16_bits_from_f32(rng.normal(0, 0.1, (V, d)).astype(np.float32)))
        self.gamma, self.beta = dev(rng.normal(1, 0.1, d).astype(np.float32)), dev(rng.normal(0, 0.1, d).astype(np.float32))
        self.h = dev_bf16(gen.bf16_bits_from_f32(rng.normal(0, 1, (M, d)).astype(np.float32)))
        self.labels = rng.integers(0, V, M).astype(np.int32)
        self.labels[::4] = -1
        self.lab = dev(self.labels)
        self.starts = dev(np.concatenate([[0], np.sort(rng.integers(0, M + 1, 5)), [M]]).astype(np.int32))
        self.adv = dev(rng.normal(0, 1, 6).astype(np.float32))
        self.head = dict(h=self.h, gamma=self.gamma, beta=self.beta, W=self.W)
        self.ws, self.ws_loss = ee.new_head_ce_grad_workspace(M, d, V), ee.new_token_loss_workspace()
        self.fwd = {k: torch.empty(n, device="cuda") for k, n in (("ce", M), ("lse", M), ("loss", 2))}
        ee.ee_head_ce(self.head, self.lab, 1e-5, out=self.fwd, workspace=self.ws)
        self.old, self.ref = (self.fwd["ce"] * 1.05).clone(), (self.fwd["ce"] * 0.9).clone()
        self.out = ee.new_policy_loss_outputs(M) if kind == "policy" else ee.new_preference_loss_outputs(M, 3)
        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        self.grad = dict(dW=torch.empty((V, d), **bf16), dgamma=torch.empty(d, **bf16), dbeta=torch.empty(d, **bf16))
        self.clipped = {k: torch.empty_like(v) for k, v in self.grad.items()}
        self.clip = ee.GradClip(self.grad.values(), out=list(self.clipped.values()))

    def step(self):
        ee = self.ee
        ee.ee_head_ce(self.head, self.lab, 1e-5, out=self.fwd, workspace=self.ws)
        if self.kind == "policy":
            ee.ee_policy_loss(self.fwd, self.lab, self.V, self.old, self.adv, ref_ce=self.ref, kl_weight=0.1, seq_start=self.starts, out=self.out,
                              workspace=self.ws_loss)
        else:
            ee.ee_preference_loss(self.fwd, self.lab, self.V, self.starts, ref_ce=self.ref, out=self.out, workspace=self.ws_loss)
        ee.ee_head_ce_grad(self.head, self.lab, 1e-5, self.fwd, dce=self.out["dce"], out=self.grad, workspace=self.ws)
        self.clip(0.01)


@pytest.mark.parametrize("kind", ["policy", "preference"])
@pytest.mark.parametrize("M,d,V", [(40, 64, 130), (300, 160, 515)])
def test_steps_then_drafts(ee, M, d, V, kind):
    m = Head(ee, M, d, V, kind)
    for _ in range(2):
        m.step()
        ref_head = dict(gamma=m.gamma.cpu().numpy(), beta=m.beta.cpu().numpy(), W=_bits(m.W).copy(), ln_eps=1e-5)
        dce = m.out["dce"].cpu().numpy()
        ref = oracle.cross_entropy(_bits(m.h), ref_head, m.labels, weights=dce)
        check(m.grad, ref, bounds(ref, ref_head["gamma"]), ("dW", "dgamma", "dbeta"))
        ce, lab, starts = m.fwd["ce"].cpu().numpy(), m.labels, m.starts.cpu().numpy()
        if kind == "policy":
            want = oracle.policy_loss(ce, m.old.cpu().numpy(), m.adv.cpu().numpy(), lab, V, m.ref.cpu().numpy(), 0.1, (0.2, 0.2), starts)
        else:
            want = oracle.preference_loss(ce, lab, V, starts, m.ref.cpu().numpy())
        assert np.abs(_np(m.out["loss"]) - want["loss"]).max() <= 2.0 ** -18 * (1 + np.abs(want["loss"]).max())
        norm = np.sqrt(sum((_np(g) ** 2).sum() for g in m.grad.values()))
        assert abs(m.clip.value.item() - norm) <= 2.0 ** -22 * norm
        factor = min(1.0, 0.01 / (norm + 1e-6))
        for k, g in m.grad.items():
            assert (np.abs(_np(m.clipped[k]) - _np(g) * factor) <= (2.0 ** -8 + 2.0 ** -20) * np.abs(_np(g)) * factor * (1 + 2.0 ** -8) + 1e-38).all()
        m.W.sub_(m.clipped["dW"])
    assert ee.ee_query_async_error(m.ws) == 0 and ee.ee_query_async_error(m.ws_loss) == 0
    serve = dict(gamma=m.gamma.cpu().numpy(), beta=m.beta.cpu().numpy(), W=_bits(m.W), ln_eps=1e-5)
    fp4 = ee.ee_head_fp4_pack(m.W, 16)
    for n in sorted({1, 9, min(M, 128), M}):
        out = ee.ee_exit_head_fp4(m.h[:n], m.gamma, m.beta, 1e-5, fp4, 2.0)
        assert_close(out, oracle.exit_head_fp4(_bits(m.h)[:n], serve, 2.0, 16), d, V, f"{n} of {M}")


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_a_captured_step_gives_what_the_eager_one_gives(ee, kind):
    m, other = Head(ee, 200, 128, 700, kind), Head(ee, 200, 128, 700, kind)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        m.step()
    for _ in range(2):                                                   # the second on weights that have changed since the capture
        graph.replay()
        other.step()
        torch.cuda.synchronize()
        for k in m.clipped:
            assert torch.equal(m.clipped[k], other.clipped[k]), k
        assert torch.equal(m.out["loss"], other.out["loss"]) and torch.equal(m.clip.value, other.clip.value)
        for t in (m, other):
            t.W.sub_(t.clipped["dW"])


@pytest.mark.parametrize("M", [3, 200])
def test_a_head_of_more_than_2_to_the_31_weights(ee, M):
    """Offsets behind 32 bits: all weights zero but one row near the end, which the rows of h point along."""
    d, V, at = 8192, 270000, 269999
    W = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    torch.manual_seed(0)
    h = torch.randn(M, d, device="cuda").bfloat16()
    W[at] = 0.01 * h[0]
    fp4 = ee.ee_head_fp4_pack(W, 32)
    assert torch.equal(ee.ee_head_fp4_unpack(fp4)[at] != 0, (ee.ee_head_fp4_unpack(ee.ee_head_fp4_pack(W[at:at + 1].contiguous(), 32)) != 0)[0])
    h[:] = h[0]
    out = ee.ee_exit_head_fp4(h, torch.ones(d, device="cuda"), torch.zeros(d, device="cuda"), 1e-5, fp4, 1.0)
    assert (out["argmax"] == at).all() and out["exit_mask"].all()
