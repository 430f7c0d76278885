"""Checks of arguments that the binding makes before anything reaches a device: no GPU needed."""
import pytest
import torch

import paper_2407_21082_b200 as ee


def _weights(kind, V=128, d=256, group=32):
    """Packed weights without a device: the checks below come before anything looks at the bytes."""
    w = object.__new__(kind)
    w.data, w.V, w.d, w.group = torch.zeros(1 << 16, dtype=torch.uint8), V, d, group
    return w


def test_the_two_4_bit_forms_are_not_taken_for_one_another():
    """A group of 32 is valid in both, and the whole-number form's bytes are enough for the other: nothing else tells them apart."""
    h = torch.zeros((2, 256), dtype=torch.bfloat16)
    gamma = beta = torch.zeros(256)
    whole, floating = _weights(ee.Q4Weights), _weights(ee.Fp4Weights)
    for call in (ee.ee_exit_head_fp4, ee.prepare_exit_head_fp4):
        with pytest.raises(TypeError, match="Fp4Weights"):
            call(h, gamma, beta, 1e-5, whole, 1.0)
    for call in (ee.ee_exit_head_q4, ee.prepare_exit_head_q4):
        with pytest.raises(TypeError, match="Q4Weights"):
            call(h, gamma, beta, 1e-5, floating, 1.0)
    with pytest.raises(TypeError):
        ee.ee_head_fp4_unpack(whole)
    with pytest.raises(TypeError):
        ee.ee_head_q4_unpack(floating)


def test_sizes_beyond_32_bits_are_invalid_and_not_cut_off():
    """2^32 + n is n to a 32-bit int: each of these had the bytes of the valid size that is left of it."""
    over = 1 << 32
    for bad in ((over + 5, 64, 16), (5, over + 64, 16), (5, 64, over + 16), (5 - over, 64, 16)):
        assert ee.ee_head_fp4_bytes(*bad) == 0
    for bad in ((over + 4, 64, 10, 16), (4, over + 64, 10, 16), (4, 64, over + 10, 16), (4, 64, 10, over + 32)):
        assert ee.ee_exit_head_fp4_workspace_bytes(*bad) == 0
    assert ee.ee_head_fp4_bytes(5, 64, 16) > 0 and ee.ee_exit_head_fp4_workspace_bytes(4, 64, 10, 16) > 0
    with pytest.raises(ee.EExitError):
        ee.Fp4Weights(torch.zeros(16, dtype=torch.uint8), over + 5, 64, 16)
