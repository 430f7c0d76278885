"""Weights, gamma, beta and packed heads that earlier work of the same stream has just written, or is still writing.

The writer is one of the library's own calls, which lets what follows it in the stream start before it has finished: ee_compact
copies a flat buffer of parameters, row by row and bit for bit, the parameters in its last rows.  The calls behind it have to give the
bits that they give for parameters that lay there long before.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

ROW = 8192                                        # bf16 words of a row of the flat buffer
PAD_ROWS = 6000                                  # in front of the parameters: some 100 MB that are copied first


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


class Flat:
    """Parameters in one flat buffer, as an optimiser holds them: `live`, and the `new` values that a step writes over it."""

    def __init__(self, ee, sizes):
        self.ee, self.at, words = ee, {}, PAD_ROWS * ROW
        for name, nbytes in sizes.items():
            self.at[name] = (words, nbytes)
            words += (nbytes + 255) // 256 * 128
        rows = (words + ROW - 1) // ROW
        self.live, self.old, self.new = (torch.zeros((rows, ROW), dtype=torch.bfloat16, device="cuda") for _ in range(3))
        self.mask = torch.zeros(rows, dtype=torch.uint8, device="cuda")
        self.out = dict(kept_idx=torch.empty(rows, dtype=torch.int32, device="cuda"), kept_count=torch.empty(1, dtype=torch.int32, device="cuda"),
                        h_out=self.live)

    def view(self, which, name, dtype, shape):
        words, nbytes = self.at[name]
        return getattr(self, which).view(-1)[words:words + nbytes // 2].view(dtype).view(shape)

    def update(self):
        self.ee.ee_compact(self.mask, self.new, out=self.out)

    def check(self, call, want, label):
        """`call` behind the update, captured and eager, from the old values every time, which a call in front of the update has read."""
        side = torch.cuda.Stream()
        torch.cuda.synchronize()                                         # `want` is there, and its workspace is free for the other stream
        with torch.cuda.stream(side):
            got = call()                                                 # nothing is set up for the first time in the capture
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                call(got)
                self.update()
                call(got)

            def eager():
                call(got)
                self.update()
                call(got)

            for turn in range(6):
                self.live.copy_(self.old)
                torch.cuda.synchronize()
                (graph.replay if turn % 2 else eager)()
                torch.cuda.synchronize()
                assert torch.equal(self.live.view(torch.int16), self.new.view(torch.int16))
                for k in want:
                    same = torch.equal(got[k], want[k])
                    assert same, (label, turn, k, int((got[k] != want[k]).sum()), got[k].numel())


def _normal(seed, *shape, scale=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return scale * torch.randn(*shape, generator=gen, device="cuda")


def _norms(flat, d):
    for which, shift in (("old", 0.5), ("new", 0.0)):
        flat.view(which, "gamma", torch.float32, (d,)).copy_(1.0 + shift + _normal(3, d, scale=0.1))
        flat.view(which, "beta", torch.float32, (d,)).copy_(shift + _normal(4, d, scale=0.1))


@pytest.mark.parametrize("M", [1, 64, 300, 1500])
@pytest.mark.parametrize("form", ["loss", "gradient"])
def test_cross_entropy_behind_an_update(ee, form, M):
    d, V = 512, 20000
    flat = Flat(ee, dict(W=V * d * 2, gamma=d * 4, beta=d * 4))
    _norms(flat, d)
    for which, seed in (("old", 5), ("new", 6)):
        flat.view(which, "W", torch.bfloat16, (V, d)).copy_(_normal(seed, V, d, scale=0.05))
    h = _normal(7, M, d).to(torch.bfloat16)
    labels = torch.randint(0, V, (M,), device="cuda", dtype=torch.int32)

    def head(which):
        return dict(h=h, gamma=flat.view(which, "gamma", torch.float32, (d,)), beta=flat.view(which, "beta", torch.float32, (d,)),
                    W=flat.view(which, "W", torch.bfloat16, (V, d)))

    ws = ee.new_head_ce_grad_workspace(M, d, V)
    fwd = {k: v.clone() for k, v in ee.ee_head_ce(head("new"), labels, 1e-5, workspace=ws).items()}
    if form == "loss":
        want = fwd
        flat.check(lambda out=None: ee.ee_head_ce(head("live"), labels, 1e-5, out=out, workspace=ws), want, M)
    else:
        want = {k: v.clone() for k, v in ee.ee_head_ce_grad(head("new"), labels, 1e-5, fwd, workspace=ws).items()}
        flat.check(lambda out=None: ee.ee_head_ce_grad(head("live"), labels, 1e-5, fwd, out=out, workspace=ws), want, M)
    assert ee.ee_query_async_error(ws) == 0


def test_steps_and_updates_in_one_graph(ee):
    """Two steps with the update of all parameters between them and no wait, against the same one by one."""
    M, d, V = 48, 256, 3001
    state = {}
    for name, t in (("W", _normal(1, V, d, scale=0.05).to(torch.bfloat16)), ("gamma", 1 + _normal(2, d, scale=0.1)), ("beta", _normal(3, d, scale=0.1))):
        state[name] = (t, t.clone())
    h = _normal(7, M, d).to(torch.bfloat16)
    labels = torch.randint(0, V, (M,), device="cuda", dtype=torch.int32)
    ws = ee.new_head_ce_grad_workspace(M, d, V)
    runs = []
    for which in (0, 1):
        p = {name: t[which] for name, t in state.items()}
        head = dict(p, h=h)
        fwd = ee.ee_head_ce(head, labels, 1e-5, workspace=ws)
        grad = ee.ee_head_ce_grad(head, labels, 1e-5, fwd, workspace=ws)

        def step(wait):
            ee.ee_head_ce(head, labels, 1e-5, out=fwd, workspace=ws)
            ee.ee_head_ce_grad(head, labels, 1e-5, fwd, out=grad, workspace=ws)
            if wait:
                torch.cuda.synchronize()
            p["W"].sub_(50 * grad["dW"])
            p["gamma"].sub_(10 * grad["dgamma"])
            p["beta"].sub_(10 * grad["dbeta"])
            if wait:
                torch.cuda.synchronize()

        torch.cuda.synchronize()
        if which == 0:
            for _ in range(6):
                step(True)
        else:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step(False)
                step(False)
            for _ in range(3):
                graph.replay()
            torch.cuda.synchronize()
        runs.append({**{k: v.clone() for k, v in fwd.items()}, **{k: v.clone() for k, v in grad.items()}, **p})
    for k in runs[0]:
        same = torch.equal(runs[0][k], runs[1][k])
        assert same, k


@pytest.mark.parametrize("d,group", [(512, 32), (2048, 128)])
@pytest.mark.parametrize("M", [1, 5, 16, 17, 64, 130])
def test_4_bit_head_behind_an_update(ee, M, d, group):
    """Streaming kernel with a warp and with all warps to a row, tensor-core kernel with one pass and with several launches."""
    V = 20000
    flat = Flat(ee, dict(packed=ee.ee_head_q4_bytes(V, d, group), gamma=d * 4, beta=d * 4))
    _norms(flat, d)

    def weights(which):
        return ee.Q4Weights(flat.view(which, "packed", torch.uint8, (-1,)), V, d, group)

    for which, seed in (("old", 5), ("new", 6)):
        ee.ee_head_q4_pack(_normal(seed, V, d, scale=0.05).to(torch.bfloat16), group, out=weights(which))
    h = _normal(7, M, d).to(torch.bfloat16)

    def head(which, out=None):
        return ee.ee_exit_head_q4(h, flat.view(which, "gamma", torch.float32, (d,)), flat.view(which, "beta", torch.float32, (d,)), 1e-5,
                                  weights(which), 7.0, out=out, workspace=ws)

    ws = ee.new_exit_head_q4_workspace(M, weights("new"))
    want = {k: v.clone() for k, v in head("new").items()}
    flat.check(lambda out=None: head("live", out), want, (M, d))
    assert ee.ee_query_async_error(ws) == 0


@pytest.mark.parametrize("M", [1, 33])
def test_packing_and_answering_in_one_graph(ee, M):
    d, V = 512, 9001
    W = _normal(1, V, d, scale=0.05).to(torch.bfloat16)
    h = _normal(2, M, d).to(torch.bfloat16)
    gamma, beta = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
    q4 = ee.ee_head_q4_pack(W, 64)
    ws = ee.new_exit_head_q4_workspace(M, q4)
    out = ee.ee_exit_head_q4(h, gamma, beta, 1e-5, q4, 7.0, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        W.mul_(0.5).add_(0.01)
        ee.ee_head_q4_pack(W, 64, out=q4)
        ee.ee_exit_head_q4(h, gamma, beta, 1e-5, q4, 7.0, out=out, workspace=ws)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        fresh = ee.ee_head_q4_pack(W, 64)
        torch.cuda.synchronize()
        want = ee.ee_exit_head_q4(h, gamma, beta, 1e-5, fresh, 7.0)
        for k in want:
            same = torch.equal(out[k], want[k])
            assert same, k
