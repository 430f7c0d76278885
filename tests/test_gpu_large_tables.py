"""Tables of more than 2^31 elements (4.4 GB): every call reaches its last rows; and calls at once on several streams.

The values of the last rows are what the same call gives on a table of those rows alone, bit for bit, or what torch gives in 64 bits.
"""
import numpy as np
import pytest
import torch

from _util import dev

pytestmark = pytest.mark.gpu
U, E = 2.0 ** -24, 2.0 ** -8
V, D = 270_000, 8192
TOP = 2 ** 31 // D + 16                                                  # the first row of a tile of 16 beyond 2^31 elements


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


@pytest.fixture(scope="module")
def table():
    gen = torch.Generator(device="cuda").manual_seed(3)
    t = torch.empty((V, D), dtype=torch.bfloat16, device="cuda")
    for r in range(0, V, 30_000):
        t[r:r + 30_000].normal_(0, 0.02, generator=gen)
    yield t
    del t
    torch.cuda.empty_cache()


def test_lookup_and_its_gradient(ee, table):
    rng = np.random.default_rng(0)
    tokens = dev(np.concatenate([[V - 1, 0, TOP, V - 1, -1, V], rng.integers(TOP, V, 40)]).astype(np.int32))
    inside = (tokens >= 0) & (tokens < V)
    rows = table[tokens.long().clamp(0, V - 1)] * inside[:, None]
    assert torch.equal(ee.ee_embed(table, tokens, 2.0), rows * 2)        # a power of two: exact
    dout = torch.randn((len(tokens), D), device="cuda").bfloat16()
    got = ee.ee_embed_grad(dout, tokens, V, 1.0)
    want = torch.zeros((V - TOP, D), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    up = inside & (tokens >= TOP)
    want.index_add_(0, tokens[up].long() - TOP, dout[up].double())
    size.index_add_(0, tokens[up].long() - TOP, dout[up].double().abs())
    assert ((got[TOP:].double() - want).abs() <= 2 * U * len(tokens) * size + E * want.abs() * (1 + U * 100)).all()
    assert torch.equal(got[0], dout[1]) and not got[1:TOP].any()


def test_packing_and_the_head_in_4_bits(ee, table):
    q4 = ee.ee_head_q4_pack(table, 64)
    last = ee.ee_head_q4_unpack(ee.ee_head_q4_pack(table[TOP - TOP % 16:].clone(), 64))
    whole = ee.ee_head_q4_unpack(q4)
    assert torch.equal(whole[TOP - TOP % 16:], last)
    gamma, beta = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    at = torch.tensor([V - 1, TOP, 17] + list(range(TOP + 1, TOP + 27)), device="cuda")
    h = (table[at].float() * 40).bfloat16()                              # a row along one of the weights' rows: that is its argmax
    for M in (3, 29):                                                    # both kernels
        out = ee.ee_exit_head_q4(h[:M], gamma, beta, 1e-5, q4, 1.0)
        assert torch.equal(out["argmax"].long(), at[:M]) and not torch.isnan(out["entropy"]).any()


def test_loss_and_gradient(ee, table):
    M = 5
    gen = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn((M, D), device="cuda", generator=gen).bfloat16()
    gamma, beta = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    labels = dev(np.array([V - 1, TOP, 3, -1, V - 2], dtype=np.int32))
    head = dict(h=h, gamma=gamma, beta=beta, W=table)
    fwd = ee.ee_head_ce(head, labels, 1e-5)
    x = h.double()
    c = x - x.mean(1, keepdim=True)
    y = (c / (c.pow(2).mean(1, keepdim=True) + 1e-5).sqrt()).float().bfloat16().double()
    z = torch.cat([y @ table[r:r + 30_000].double().T for r in range(0, V, 30_000)], 1)
    mag = max(float((y.abs() @ table[r:r + 30_000].double().abs().T).max()) for r in range(0, V, 30_000))
    dz = 2 * U * D * mag                                                 # D additions in fp32, each off by 2u of the running magnitude
    lse = torch.logsumexp(z, 1)
    off = dz + 2.0 ** -21 + 2 * U * (64 + V / 64) + 2 * U * lse.abs()
    on = labels >= 0
    ce = torch.where(on, lse - z.gather(1, labels.long().clamp(min=0)[:, None])[:, 0], 0.0)
    assert ((fwd["lse"].double() - lse).abs() <= off).all() and ((fwd["ce"].double() - ce).abs() <= off + dz + 2 * U * ce.abs()).all()
    out = ee.ee_head_ce_grad(head, labels, 1e-5, fwd)
    G = torch.softmax(z, 1)
    G[torch.arange(M, device="cuda")[on], labels[on].long()] -= 1
    G = G * on[:, None] / on.sum()
    # dW's last rows: G is off by r of the softmax and by one rounding to bf16; the sum over five rows, and its rounding
    r = dz + off[:, None] + 2.0 ** -21
    dG = (r * torch.softmax(z, 1) / on.sum() * on[:, None]) * (1 + E) + E * G.abs() * (1 + 8 * U)
    want, bound = G[:, TOP:].T @ y, dG[:, TOP:].T @ y.abs() + 2 * U * (M + 2) * (G[:, TOP:].abs().T @ y.abs())
    bound = bound * (1 + E) + E * want.abs() + 1e-38
    assert ((out["dW"][TOP:].double() - want).abs() <= bound).all()
    assert not out["dh"][3].any() and torch.isfinite(out["dh"].float()).all()


def test_calls_at_once_on_several_streams(ee):
    d, v = 256, 3000
    gen = torch.Generator(device="cuda").manual_seed(5)
    W = (torch.randn((v, d), device="cuda", generator=gen) * 0.05).bfloat16()
    gamma, beta = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
    q4 = ee.ee_head_q4_pack(W, 64)
    h = torch.randn((200, d), device="cuda", generator=gen).bfloat16()
    tokens = torch.randint(0, v, (200,), device="cuda", dtype=torch.int32, generator=gen)
    head = dict(h=h, gamma=gamma, beta=beta, W=W)

    def ce(ws):
        f = ee.ee_head_ce(head, tokens, 1e-5, workspace=ws)
        return {**f, **ee.ee_head_ce_grad(head, tokens, 1e-5, f, workspace=ws)}

    jobs = [(lambda ws: ee.ee_exit_head_q4(h[:7], gamma, beta, 1e-5, q4, 1.0, workspace=ws), lambda: ee.new_exit_head_q4_workspace(7, q4)),
            (lambda ws: ee.ee_exit_head_q4(h, gamma, beta, 1e-5, q4, 1.0, workspace=ws), lambda: ee.new_exit_head_q4_workspace(200, q4)),
            (lambda ws: dict(g=ee.ee_embed_grad(h, tokens, v, 0.5, workspace=ws)), lambda: ee.new_embed_grad_workspace(200, d, v)),
            (ce, lambda: ee.new_head_ce_grad_workspace(200, d, v))]
    want = [job(space()) for job, space in jobs]
    streams, spaces = [torch.cuda.Stream() for _ in range(8)], [jobs[i % 4][1]() for i in range(8)]
    torch.cuda.synchronize()
    got = [[] for _ in streams]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(jobs[i % 4][0](spaces[i]))
    torch.cuda.synchronize()
    for i, runs in enumerate(got):
        for run in runs:
            for k in run:
                assert torch.equal(run[k], want[i % 4][k]), (i % 4, k)
