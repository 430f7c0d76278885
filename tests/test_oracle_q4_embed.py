"""Pins of the 4-bit and embedding oracles."""
import numpy as np

import gen
import oracle


def _bits(x):
    return gen.bf16_bits_from_f32(np.asarray(x, dtype=np.float32))


def test_quantisation_by_hand():
    w = np.zeros((2, 32), np.float32)
    w[0, :6] = [7.0, -7.0, 3.5, 2.5, -0.49, 1.5]          # scale exactly 1: ties go to the even number
    q, s = oracle.q4_quantise(_bits(w), 32)
    assert s[0, 0] == 1.0 and list(q[0, :6]) == [7, -7, 4, 2, 0, 2]      # (-0.49 is no tie)
    assert s[1, 0] == 0.0 and not q[1].any()
    assert np.array_equal(oracle.bf16_decode(oracle.q4_values(_bits(w), 32))[0, :6], [7, -7, 4, 2, 0, 2])


def test_quantisation_error_is_at_most_half_a_step():
    rng = np.random.default_rng(0)
    W = _bits(rng.normal(0, 0.02, (50, 256)))
    for group in (32, 64, 128):
        q, s = oracle.q4_quantise(W, group)
        step = np.repeat(s, group, axis=1)
        assert np.abs(q).max() <= 7 and (np.abs(q).reshape(50, -1, group).max(axis=2) == 7).all()
        # half a step, and what the scale's rounding (2^-8 of it) takes off the largest magnitudes
        assert (np.abs(q * step - oracle.bf16_decode(W)) <= step * (0.5 + 7 * 2.0 ** -8)).all()
        v = oracle.bf16_decode(oracle.q4_values(W, group))
        assert (np.abs(v - q * step) <= np.abs(q * step) * 2.0 ** -8).all()


def test_embedding_by_loops():
    rng = np.random.default_rng(1)
    table, dout = _bits(rng.normal(0, 1, (7, 8))), _bits(rng.normal(0, 1, (5, 8)))
    tokens = np.array([3, -1, 3, 6, 7])
    out = oracle.embed(table, tokens, 2.5)
    grad, size, count = oracle.embed_grad(dout, tokens, 7, 2.5)
    t, g = oracle.bf16_decode(table), oracle.bf16_decode(dout)
    assert np.array_equal(out[0], t[3] * 2.5) and not out[1].any() and not out[4].any()
    assert np.allclose(grad[3], 2.5 * (g[0] + g[2]), atol=1e-15) and np.array_equal(grad[6], 2.5 * g[3])
    assert list(count) == [0, 0, 0, 2, 0, 0, 1] and not grad[[0, 1, 2, 4, 5]].any()
    # the gradient is the transpose of the lookup: <dout, lookup(table)> = <grad, table>
    assert abs((g * out).sum() - (grad * t).sum()) < 1e-12
