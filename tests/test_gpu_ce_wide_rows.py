"""ee_head_ce on wide rows: a logit is summed in parts, because the tensor core's accumulator cuts off what falls below its last bit.

The logits are built so that an accumulator that starts with the largest term would lose all the others: y is 1 everywhere (gamma = 0, beta = 1), every
weight row is 16 in its first column and 9.4e-8 in the rest, so that the 16 products of one step add 1.5e-6, less than a step of 16 in
fp32 (2^-19).  Bound: the first part, up to 1024 columns, may lose two steps of 16 (the truncation and the alignment of the products) in each of its
64 additions, the parts' sums a rounding each (2^-19 for up to eight), and ln sum exp what test_gpu_ce.py allows it.
"""
import numpy as np
import pytest
import torch

import oracle
from _util import dev, dev_bf16
from gen import bf16_bits_from_f32

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


@pytest.mark.parametrize("M", [1, 64, 130, 600])
@pytest.mark.parametrize("d", [4096, 5000, 8192])
def test_small_terms_behind_a_large_one_are_not_lost(ee, M, d):
    V = 500
    W = np.full((V, d), 1.5e-6 / 16, np.float32)
    W[:, 0] = 16.0
    bits = bf16_bits_from_f32(W)
    z = oracle.bf16_decode(bits[0]).sum()
    head = dict(h=dev_bf16(bf16_bits_from_f32(np.random.default_rng(1).normal(0, 1, (M, d)).astype(np.float32))), gamma=torch.zeros(d, device="cuda"),
                beta=torch.ones(d, device="cuda"), W=dev_bf16(bits))
    labels = dev(np.arange(M, dtype=np.int32) % V)
    fwd = ee.ee_head_ce(head, labels, 1e-5)
    lse = z + np.log(V)
    bound = 64 * 2 * 2.0 ** -19 + 8 * 2.0 ** -19 + 2.0 ** -21 + 2 * U * (64 + V / 64) + 2 * U * lse
    assert (d / 16 - 64) * 1.4e-6 > bound - 5e-5                         # what one accumulator for all of it would lose, about
    err = np.abs(fwd["lse"].cpu().numpy().astype(np.float64) - lse).max()
    assert err <= bound, (err, bound)
    # the gradient's logits are the same: all columns alike but the label's
    grad = ee.ee_head_ce_grad(head, labels, 1e-5, fwd, dce=torch.ones(M, device="cuda"))
    db = grad["dbeta"].float().cpu().numpy().astype(np.float64)
    assert (np.abs(db) <= 16 * M * 2.0 ** -8 * (2 + M * 2.0 ** -8)).all()       # every row's G sums to zero up to its roundings, times W <= 16


@pytest.mark.parametrize("M,d,V", [(64, 2048, 50304), (300, 1536, 20011), (300, 2048, 50304), (1500, 1088, 20011), (520, 4096, 20011), (520, 2560, 20011)])
def test_many_tiles_of_even_and_odd_numbers_of_parts(ee, M, d, V):
    """Several tiles to a CTA, whose four groups of columns meet in shared memory at every one; against the same in 64 bits, and the same
    bits every time.  lse: dz = 2 u d max_v sum |w y| and what test_gpu_ce.py allows the sum of exponentials."""
    rng = torch.Generator(device="cuda").manual_seed(d)
    W = (0.05 * torch.randn(V, d, generator=rng, device="cuda")).to(torch.bfloat16)
    h = torch.randn(M, d, generator=rng, device="cuda").to(torch.bfloat16)
    labels = torch.randint(0, V, (M,), generator=rng, device="cuda").to(torch.int32)
    head = dict(h=h, gamma=torch.ones(d, device="cuda"), beta=torch.zeros(d, device="cuda"), W=W)
    x = h.double()
    c = x - x.mean(1, keepdim=True)
    y = (c * torch.rsqrt((c * c).mean(1, keepdim=True) + 1e-5)).float().to(torch.bfloat16).double()
    z = y @ W.double().t()
    lse = torch.logsumexp(z, 1)
    ce = lse - z.gather(1, labels.long()[:, None])[:, 0]
    dz = 2 * U * d * (y.abs() @ W.double().abs().t()).amax(1)
    dlse = dz + 2.0 ** -21 + 2 * U * (64 + V / 64) + 2 * U * lse.abs()
    first = None
    for _ in range(20):
        got = ee.ee_head_ce(head, labels, 1e-5)
        assert ((got["lse"].double() - lse).abs() <= dlse).all()
        assert ((got["ce"].double() - ce).abs() <= dlse + dz + 2 * U * ce.abs()).all()
        first = first or got
        same = torch.equal(got["lse"], first["lse"]) and torch.equal(got["ce"], first["ce"])
        assert same
