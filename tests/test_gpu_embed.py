"""ee_embed and ee_embed_grad against the oracle.

Bounds (u = 2^-24, e = 2^-8): the lookup is one fp32 product and one rounding to bf16, both reproduced exactly here.  A sum of
k fp32 terms in any order is off by at most k u times the sum of magnitudes (one rounding each), the scale adds one
more rounding, bf16 output e of the result, accumulation one more of each.
"""
import numpy as np
import pytest
import torch

import gen
import oracle
from _util import dev, dev_bf16

pytestmark = pytest.mark.gpu
U, E = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _rand_bits(rng, *shape, std=1.0):
    return gen.bf16_bits_from_f32(rng.normal(0, std, shape).astype(np.float32))


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("n,d,V", [(1, 8, 1), (5, 72, 30), (33, 1024, 500), (300, 2560, 2000), (10000, 16, 50304), (3, 8192, 9)])
def test_lookup_is_exact(ee, n, d, V):
    rng = np.random.default_rng(n)
    table = _rand_bits(rng, V, d, std=0.02)
    tokens = rng.integers(0, V, n).astype(np.int32)
    if n > 2:
        tokens[:3] = [-1, V, V - 1]
    scale = np.float32(np.sqrt(d))
    out = ee.ee_embed(dev_bf16(table), dev(tokens), float(scale))
    # the fp32 product of the definition, then one rounding
    prod = (gen.f32_from_bf16_bits(table) * scale)[np.clip(tokens, 0, V - 1)]
    want = np.where(((tokens >= 0) & (tokens < V))[:, None], gen.bf16_bits_from_f32(prod), 0)
    assert np.array_equal(out.view(torch.int16).cpu().numpy().view(np.uint16), want)
    ref = oracle.embed(table, tokens, scale)
    assert (np.abs(_np(out) - ref) <= np.abs(ref) * (E + 2 * U)).all()
    wide = torch.full((n + 1, d + 16), 3.0, dtype=torch.bfloat16, device="cuda")
    ee.ee_embed(dev_bf16(table), dev(tokens), float(scale), out=wide[:n, 8:8 + d])
    assert torch.equal(wide[:n, 8:8 + d], out) and (wide[n] == 3).all() and (wide[:, :8] == 3).all() and (wide[:, 8 + d:] == 3).all()


def _tokens(rng, kind, n, V):
    if kind == "one":
        t = np.full(n, V - 1)
    elif kind == "zipf":
        t = np.minimum(V - 1, np.exp(rng.random(n) * np.log(V)).astype(np.int64) - 1)
    elif kind == "two":
        t = np.where(rng.random(n) < 0.5, 0, V - 1)
    elif kind == "none":
        t = rng.choice([-1, V, -2 ** 31, 2 ** 31 - 1], n)
    else:
        t = rng.integers(0, V, n)
        t[rng.random(n) < 0.2] = -1
    return t.astype(np.int32)


GRADS = [(1, 8, 1, "one"), (1, 72, 50, "mixed"), (7, 64, 3, "mixed"), (8, 64, 300, "one"), (9, 64, 300, "one"), (257, 520, 700, "zipf"),
         (1000, 1024, 90, "two"), (4096, 40, 50304, "zipf"), (16384, 64, 65535, "zipf"), (16384, 16, 65536, "mixed"), (16385, 64, 5000, "zipf"),
         (40000, 24, 900, "one"), (40000, 8, 50304, "mixed"), (500, 8, 262143, "mixed"), (500, 8, 262144, "mixed"), (3000, 8, 300001, "zipf"),
         (100, 8192, 20, "zipf"), (777, 64, 100, "none"), (20000, 64, 100, "none")]


@pytest.mark.parametrize("n,d,V,kind", GRADS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradient_matches_the_oracle(ee, n, d, V, kind, dtype):
    rng = np.random.default_rng(n + d + V)
    dout, tokens, scale = _rand_bits(rng, n, d), _tokens(rng, kind, n, V), np.float32(1.7)
    ref, size, count = oracle.embed_grad(dout, tokens, V, scale)
    bound = (count[:, None] + 2) * U * size * 2
    if dtype == torch.bfloat16:
        bound = bound + E * (np.abs(ref) + bound)
    out = ee.ee_embed_grad(dev_bf16(dout), dev(tokens), V, float(scale), dtype=dtype)
    assert (np.abs(_np(out) - ref) <= bound).all()
    again = ee.ee_embed_grad(dev_bf16(dout), dev(tokens), V, float(scale), dtype=dtype)
    assert torch.equal(out, again)                                       # a fixed order
    # adding to what is there: one rounding, other rows untouched
    old_bits = _rand_bits(rng, V, d)
    old = dev_bf16(old_bits).to(dtype)
    got = ee.ee_embed_grad(dev_bf16(dout), dev(tokens), V, float(scale), out=old.clone(), accumulate=True)
    want = ref + oracle.bf16_decode(old_bits)
    eps = E if dtype == torch.bfloat16 else U
    assert (np.abs(_np(got) - want) <= bound + eps * (np.abs(want) + bound) + U * np.abs(want) * 2).all()
    rest = torch.from_numpy(np.flatnonzero(count == 0)).cuda()
    assert torch.equal(got[rest], old[rest])


def test_gradient_of_strided_rows_with_not_a_number_in_rows_left_out(ee):
    n, d, V = 600, 136, 50
    rng = np.random.default_rng(8)
    dout, tokens = _rand_bits(rng, n, d), _tokens(rng, "mixed", n, V)
    want = ee.ee_embed_grad(dev_bf16(dout), dev(tokens), V, 0.5)
    wide = torch.full((n, d + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + d] = dev_bf16(dout)
    wide[torch.from_numpy(tokens < 0).cuda()] = float("nan")
    assert torch.equal(ee.ee_embed_grad(wide[:, 8:8 + d], dev(tokens), V, 0.5), want)


def test_gradient_against_differences_of_the_lookup(ee):
    """<dout, lookup(table)> is linear in the table: its difference for a step in one element is the gradient's element."""
    n, d, V = 50, 16, 12
    rng = np.random.default_rng(9)
    dout, tokens = _rand_bits(rng, n, d), _tokens(rng, "mixed", n, V)
    grad = ee.ee_embed_grad(dev_bf16(dout), dev(tokens), V, 2.0, dtype=torch.float32)
    table = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    for v, j in [(0, 0), (5, 7), (11, 15)]:
        table.zero_()
        table[v, j] = 1.0
        diff = float((dev_bf16(dout).double() * ee.ee_embed(table, dev(tokens), 2.0).double()).sum())
        assert abs(diff - float(grad[v, j])) <= 1e-5 * (1 + abs(diff))


@pytest.mark.parametrize("n", [700, 17000])
def test_captured_beside_an_eager_call(ee, n):
    d, V = 64, 3000
    rng = np.random.default_rng(10)
    dout, tokens = dev_bf16(_rand_bits(rng, n, d)), dev(_tokens(rng, "zipf", n, V))
    want = ee.ee_embed_grad(dout, tokens, V).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call = ee.prepare_embed_grad(dout, tokens, V, workspace=ee.new_embed_grad_workspace(n, d, V))
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    call.out.fill_(float("nan"))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.replay()
        graph.replay()
    eager = ee.ee_embed_grad(dout, tokens, V)
    torch.cuda.synchronize()
    assert torch.equal(call.out, want) and torch.equal(eager, want)


@pytest.mark.parametrize("n,d,V,kind", [(1, 8, 1, "one"), (300, 64, 50, "zipf"), (5000, 24, 900, "two"), (17000, 64, 900, "mixed")])
def test_what_the_workspace_held_does_not_matter(ee, n, d, V, kind):
    rng = np.random.default_rng(n)
    dout, tokens = dev_bf16(_rand_bits(rng, n, d)), dev(_tokens(rng, kind, n, V))
    ws = ee.new_embed_grad_workspace(n, d, V)
    results = []
    for junk in (0, 255):
        ws.fill_(junk)
        results.append(ee.ee_embed_grad(dout, tokens, V, workspace=ws, out=torch.full((V, d), float("nan"), device="cuda")))
    assert torch.isfinite(results[1]).all() and torch.equal(results[0], results[1])


def test_nothing_to_look_up(ee):
    table = torch.ones((5, 16), dtype=torch.bfloat16, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert ee.ee_embed(table, none).shape == (0, 16)
    dout = torch.empty((0, 16), dtype=torch.bfloat16, device="cuda")
    assert not ee.ee_embed_grad(dout, none, 5).any()
    assert torch.equal(ee.ee_embed_grad(dout, none, 5, out=table.clone(), accumulate=True), table)


def test_refusals(ee):
    table = torch.ones((5, 16), dtype=torch.bfloat16, device="cuda")
    tokens = torch.zeros(4, dtype=torch.int32, device="cuda")
    dout = torch.ones((4, 16), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        ee.ee_embed(table, tokens.long())
    with pytest.raises(ValueError):
        ee.ee_embed(table[:, :8], tokens)
    with pytest.raises(ValueError):
        ee.ee_embed(table, tokens, out=torch.empty((3, 16), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError):
        ee.ee_embed(table.float(), tokens)
    with pytest.raises(ee.EExitError) as e:
        ee.ee_embed(torch.ones((5, 12), dtype=torch.bfloat16, device="cuda"), tokens)
    assert e.value.code == 2
    with pytest.raises(ValueError):
        ee.ee_embed_grad(dout, tokens[:3], 5)
    with pytest.raises(ValueError):
        ee.ee_embed_grad(dout, tokens, 5, dtype=torch.float16)
    with pytest.raises(ValueError):
        ee.ee_embed_grad(dout, tokens, 5, accumulate=True)
    with pytest.raises(ValueError):
        ee.ee_embed_grad(dout, tokens, 5, out=torch.empty((4, 16), device="cuda"))
    with pytest.raises(ee.EExitError) as e:
        ee.ee_embed_grad(dout, tokens, 5, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 4


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 127, 511, 512, 513])
@pytest.mark.parametrize("kind", ["one", "two", "none", "mixed"])
def test_lists_about_the_length_that_is_not_sorted(ee, n, kind):
    """Exact against the oracle's sum: values of whole numbers up to 8 in magnitude, so every fp32 sum of 513 is exact in any order."""
    d, V = 1032, 700                                                     # 129 vectors: one more than a CTA takes
    rng = np.random.default_rng(n)
    dout = gen.bf16_bits_from_f32(rng.integers(-8, 9, (n, d)).astype(np.float32))
    tokens = _tokens(rng, kind, n, V)
    ref, _, count = oracle.embed_grad(dout, tokens, V, np.float32(1.0))
    out = ee.ee_embed_grad(dev_bf16(dout), dev(tokens), V, 1.0, dtype=torch.float32, out=torch.full((V, d), float("nan"), device="cuda"))
    assert np.array_equal(_np(out), ref)
    old = torch.full((V, d), 3.0, device="cuda")
    ee.ee_embed_grad(dev_bf16(dout), dev(tokens), V, 1.0, out=old, accumulate=True)
    assert np.array_equal(_np(old), ref + 3.0)


def test_a_short_list_behind_work_that_writes_it(ee):
    """The rows and the tokens are read while the table is being cleared: what an earlier kernel of the stream wrote must be there."""
    n, d, V = 300, 520, 40000
    rng = np.random.default_rng(1)
    outs, wants = [], []
    src = [dev_bf16(_rand_bits(rng, n, d)) for _ in range(6)]
    toks = [dev(_tokens(rng, "mixed", n, V)) for _ in range(6)]
    for s, t in zip(src, toks):
        torch.cuda.synchronize()
        wants.append(ee.ee_embed_grad(s, t, V, 2.0))
    torch.cuda.synchronize()
    rows, tok = torch.empty_like(src[0]), torch.empty_like(toks[0])
    for s, t in zip(src, toks):
        rows.copy_(s)
        tok.copy_(t)
        outs.append(ee.ee_embed_grad(rows, tok, V, 2.0))
    for a, b in zip(outs, wants):
        assert torch.equal(a, b)
