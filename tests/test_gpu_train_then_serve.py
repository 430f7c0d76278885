"""The operators of training and of serving with 4 bits, one after the other as a program uses them: a model whose embedding is
tied to its head learns for a few steps, its table is packed, and rows are answered one by one and in batches.

Bounds: those of the single operators, carried through.  The table's gradient is dW (its bound has the rounding to bf16) plus, for a
row of the table, the rows of dh of its tokens times the scale: scale x (the sum of dh's bounds + (k + 2) 2u of the sum of
magnitudes for k tokens), and one rounding of the total to bf16.
"""
import numpy as np
import pytest
import torch

import gen
import oracle
from _util import assert_head_matches, dev, dev_bf16, oracle_head
from test_gpu_ce import E, U, bounds, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _bits(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Tied:
    """A table that is embedding and head, and one training step through the operators, in buffers of its own."""

    def __init__(self, ee, M, d, V, seed=5):
        self.ee, self.M, self.d, self.V, self.scale = ee, M, d, V, 4.0
        rng = np.random.default_rng(seed)
        self.table = dev_bf16(gen.bf16_bits_from_f32(rng.normal(0, 0.05, (V, d)).astype(np.float32)))
        self.gamma = dev(rng.normal(1, 0.1, d).astype(np.float32))
        self.beta = dev(rng.normal(0, 0.1, d).astype(np.float32))
        self.tokens = rng.integers(0, V, M).astype(np.int32)
        self.labels = ((self.tokens.astype(np.int64) * 7 + 3) % V).astype(np.int32)
        self.tokens[M // 2:] = self.tokens[0]                            # one token in half the rows
        self.labels[1::5] = -1
        self.labels[0] = V - 1
        self.tok, self.lab = dev(self.tokens), dev(self.labels)
        self.h = torch.empty((M, d), dtype=torch.bfloat16, device="cuda")
        self.head = dict(h=self.h, gamma=self.gamma, beta=self.beta, W=self.table)
        self.ws = ee.new_head_ce_grad_workspace(M, d, V)
        self.ws_embed = ee.new_embed_grad_workspace(M, d, V)
        self.fwd = {k: torch.empty(n, device="cuda") for k, n in (("ce", M), ("lse", M), ("loss", 2))}
        self.grad = {"dh": torch.empty_like(self.h), "dW": torch.empty_like(self.table)}
        self.dtable = torch.empty_like(self.table)

    def step(self):
        ee = self.ee
        ee.ee_embed(self.table, self.tok, self.scale, out=self.h)
        ee.ee_head_ce(self.head, self.lab, 1e-5, out=self.fwd, workspace=self.ws)
        ee.ee_head_ce_grad(self.head, self.lab, 1e-5, self.fwd, out=self.grad, workspace=self.ws)
        self.dtable.copy_(self.grad["dW"])
        ee.ee_embed_grad(self.grad["dh"], self.tok, self.V, self.scale, out=self.dtable, accumulate=True, workspace=self.ws_embed)


@pytest.mark.parametrize("M,d,V", [(1, 32, 40), (67, 96, 515), (300, 320, 1003)])
def test_training_steps_then_answers_in_4_bits(ee, M, d, V):
    m = Tied(ee, M, d, V)
    for _ in range(3):
        m.step()
        h_bits = _bits(m.h)
        table = _bits(m.table).copy()
        at = gen.f32_from_bf16_bits(table)[m.tokens] * np.float32(m.scale)
        assert np.array_equal(h_bits, gen.bf16_bits_from_f32(at))
        head = dict(gamma=m.gamma.cpu().numpy(), beta=m.beta.cpu().numpy(), W=table, ln_eps=1e-5)
        ref = oracle.cross_entropy(h_bits, head, m.labels)
        bnd = bounds(ref, head["gamma"])
        check(m.fwd, ref, bnd, ("ce", "lse"))
        check(m.grad, ref, bnd, ("dh", "dW"))
        want, off, size, count = ref["dW"].copy(), bnd["dW"].copy(), np.zeros((V, d)), np.zeros(V)
        np.add.at(want, m.tokens, m.scale * ref["dh"])
        np.add.at(off, m.tokens, m.scale * bnd["dh"])
        np.add.at(size, m.tokens, m.scale * (np.abs(ref["dh"]) + bnd["dh"]))
        np.add.at(count, m.tokens, 1)
        off = off + (count[:, None] + 2) * 2 * U * (size + np.abs(ref["dW"]) + bnd["dW"])
        off = off + E * (np.abs(want) + off)
        assert (np.abs(_np(m.dtable) - want) <= off).all()
        m.table.copy_((m.table.float() - 0.5 * m.dtable.float()).to(torch.bfloat16))
    assert ee.ee_query_async_error(m.ws) == 0

    q4 = ee.ee_head_q4_pack(m.table, 32)
    table = _bits(m.table)
    serve = dict(gamma=m.gamma.cpu().numpy(), beta=m.beta.cpu().numpy(), W=oracle.q4_values(table, 32), ln_eps=1e-5)
    for n in sorted({1, min(M, 16), min(M, 40), M}):                     # single tokens, both kernels, several launches
        h = ee.ee_embed(m.table, m.tok[:n].contiguous(), m.scale)
        out = ee.ee_exit_head_q4(h, m.gamma, m.beta, 1e-5, q4, 2.0)
        assert_head_matches(out, oracle_head(_bits(h), serve, 2.0), label=f"{n} of {M}")


def test_a_captured_step_gives_what_the_eager_one_gives(ee):
    m = Tied(ee, 200, 128, 700)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        m.step()
    other = Tied(ee, 200, 128, 700)
    for _ in range(2):                                                   # the second on a table that has changed since the capture
        graph.replay()
        other.step()
        torch.cuda.synchronize()
        assert torch.equal(m.dtable, other.dtable) and torch.equal(m.fwd["loss"], other.fwd["loss"])
        for t in (m, other):
            t.table.sub_((0.5 * t.dtable.float()).to(torch.bfloat16))


@pytest.mark.parametrize("M", [1, 5, 16, 17, 64])
def test_entropies_of_nearly_certain_rows_keep_their_digits(ee, M):
    """H = ln s - t / s with s just above 1.  With every difference of two logits off by at most x, to first order
    |dH| <= sum p |ln p + H| x <= 2 H x; x = 2 dz with dz = 2u d sum |w y| (fp32 sums) + 2u |z| (the difference to the maximum and its
    product), and 2^-21 + 2u (64 + V / 64) relative for the exponentials and their sums, twice (once for t)."""
    d, V, group = 64, 200, 32
    rng = np.random.default_rng(12)
    W = rng.normal(0, 0.3, (V, d)).astype(np.float32)
    w_bits = gen.bf16_bits_from_f32(W)
    W4 = oracle.q4_values(w_bits, group)
    vals = oracle.bf16_decode(W4)
    h = vals[rng.integers(0, V, M)] * 3 + rng.normal(0, 0.1, (M, d))
    h_bits = gen.bf16_bits_from_f32(h.astype(np.float32))
    gamma, beta = np.full(d, 1.2, np.float32), np.zeros(d, np.float32)
    ref = oracle.cross_entropy(h_bits, dict(gamma=gamma, beta=beta, W=W4, ln_eps=1e-5), np.zeros(M, np.int32))
    z = ref["y"] @ vals.T
    dz = z - z.max(1, keepdims=True)
    e = np.exp(dz)
    rest = e.sum(1) - 1.0                                                # in 64 bits the 1 costs nothing here
    H = np.log1p(rest) - (e * dz).sum(1) / (1.0 + rest)
    x = 2 * (2 * U * d * (np.abs(ref["y"]) @ np.abs(vals).T).max(1) + 2 * U * np.abs(z).max(1))
    bound = H * (2 * x + 2 * (2.0 ** -21 + 2 * U * (64 + V / 64)))
    got = ee.ee_exit_head_q4(dev_bf16(h_bits), dev(gamma), dev(beta), 1e-5, ee.ee_head_q4_pack(dev_bf16(w_bits), group), 0.5)
    assert H.max() < 0.05 and H.min() < 1e-4                             # what the test is about
    assert (np.abs(_np(got["entropy"]) - H) <= bound).all()
    assert got["exit_mask"].all()


def test_any_label_outside_the_vocabulary_marks_a_row(ee):
    """The extreme ones too, in every piece of the vocabulary."""
    M, d, V = 600, 8, 140000                                             # G is more than one piece holds
    rng = np.random.default_rng(2)
    head = dict(h=dev_bf16(gen.bf16_bits_from_f32(rng.normal(0, 1, (M, d)).astype(np.float32))), gamma=torch.ones(d, device="cuda"),
                beta=torch.zeros(d, device="cuda"), W=dev_bf16(gen.bf16_bits_from_f32(rng.normal(0, 0.3, (V, d)).astype(np.float32))))
    labels = rng.integers(0, V, M).astype(np.int32)
    labels[::3] = -1
    extreme = labels.copy()
    extreme[::3] = rng.choice([-2 ** 31, -2 ** 31 + 1, 2 ** 31 - 1, V, -V, -1], len(labels[::3]))
    got = []
    for lab in (labels, extreme):
        fwd = ee.ee_head_ce(head, dev(lab), 1e-5)
        got.append({**fwd, **ee.ee_head_ce_grad(head, dev(lab), 1e-5, fwd)})
    for k in got[0]:
        assert torch.equal(got[0][k], got[1][k]), k
