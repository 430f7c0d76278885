"""ee_embed_grad where lists are sorted (more than 512 tokens): the widest tokens the cluster's sort packs into a word, the first ones it does
not, and calls at once on several streams.  Bounds as in test_gpu_embed.py."""
import numpy as np
import pytest
import torch

import oracle
from _util import dev, dev_bf16
from test_gpu_embed import E, U, _np, _rand_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _tokens(rng, n, V):
    """All over the table, its two ends and what lies just outside it among them, some in long runs."""
    t = rng.integers(0, V, n)
    t[rng.random(n) < 0.3] = V - 1
    t[rng.random(n) < 0.1] = 0
    t[rng.random(n) < 0.1] = V
    t[rng.random(n) < 0.1] = rng.choice([-1, V + 1, -2 ** 31, 2 ** 31 - 1])
    t[[0, n - 1, n // 2]] = [V - 1, V - 2 if V > 1 else 0, V]
    return t.astype(np.int32)


@pytest.mark.parametrize("n", [513, 600, 2048, 2049, 16383, 16384, 16385])
@pytest.mark.parametrize("V", [1, 255, 256, 65535, 65536, 262143, 262144])
def test_tables_on_both_sides_of_what_a_word_holds(ee, n, V):
    d = 8
    rng = np.random.default_rng(n * 3 + V)
    dout, tokens, scale = _rand_bits(rng, n, d), _tokens(rng, n, V), np.float32(1.7)
    ref, size, count = oracle.embed_grad(dout, tokens, V, scale)
    bound = (count[:, None] + 2) * U * size * 2
    ws = ee.new_embed_grad_workspace(n, d, V)
    for junk in (0, 255):
        ws.fill_(junk)
        out = ee.ee_embed_grad(dev_bf16(dout), dev(tokens), V, float(scale), dtype=torch.float32, workspace=ws)
        assert (np.abs(_np(out) - ref) <= bound).all()
    out = ee.ee_embed_grad(dev_bf16(dout), dev(tokens), V, float(scale), workspace=ws)
    assert (np.abs(_np(out) - ref) <= bound + E * (np.abs(ref) + bound)).all()


@pytest.mark.parametrize("accumulate", [False, True])
def test_calls_at_once_on_eight_streams(ee, accumulate):
    """Sorted in a cluster and in memory, each with a workspace and a table of its own."""
    rng = np.random.default_rng(5)
    jobs = []
    for i, (n, d, V) in enumerate([(600, 64, 5000), (16384, 64, 50304), (3000, 264, 300), (16385, 64, 4000), (9000, 8, 262143), (513, 1032, 900),
                                   (20000, 16, 70000), (12345, 32, 65536)]):
        dout, tokens = dev_bf16(_rand_bits(rng, n, d)), dev(_tokens(rng, n, V))
        old = dev_bf16(_rand_bits(rng, V, d))
        want = old.clone()
        ee.ee_embed_grad(dout, tokens, V, 0.5, out=want, accumulate=accumulate)
        jobs.append((dout, tokens, V, old, want, ee.new_embed_grad_workspace(n, d, V), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(4):
        got = [job[3].clone() for job in jobs]
        torch.cuda.synchronize()
        for out, (dout, tokens, V, old, want, ws, stream) in zip(got, jobs):
            with torch.cuda.stream(stream):
                ee.ee_embed_grad(dout, tokens, V, 0.5, out=out, accumulate=accumulate, workspace=ws)
        torch.cuda.synchronize()
        for out, job in zip(got, jobs):
            same = torch.equal(out, job[4])
            assert same, job[0].shape
