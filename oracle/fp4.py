"""fp64 CPU oracle for heads held in microscaled 4-bit floating point (see include/eexit.h, "Heads held in microscaled 4-bit floating point").

TEST INFRASTRUCTURE ONLY (see oracle/exit_head.py).  Shares no code with the CUDA sources.
"""
from __future__ import annotations

import numpy as np

from .ce_loss import _rows, bf16_by_f32
from .exit_head import bf16_decode, exit_decision, softmax_stats

ELEMENTS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _floor_log2(t):
    return np.frexp(np.where(t > 0, t, 1.0))[1] - 1


def round_e2m1(a):
    """Nearest element, ties to the even code, at most 6."""
    m = np.abs(a)
    middles = (ELEMENTS[1:] + ELEMENTS[:-1]) / 2
    code = np.searchsorted(middles, m, side="left")              # a middle counts to the code below it ...
    odd = (code % 2 == 1) & (m == middles[np.minimum(code, 6)])  # ... unless that is odd
    return np.copysign(ELEMENTS[np.where(odd, code + 1, code)], a)


def round_e4m3(a):
    """Nearest number of four exponent and three mantissa bits (positive, below 448), ties to even."""
    step = np.ldexp(1.0, np.maximum(_floor_log2(a), -6) - 3)
    return np.rint(a / step) * step


def quantise(x, group: int, by_row: bool):
    """Elements [n, d] and scales [n, d / group] of a matrix of bf16 values (fp64 array)."""
    n, d = x.shape
    g = np.asarray(x, dtype=np.float64).reshape(n, d // group, group)
    top = np.abs(g).max(axis=2)
    if group == 32:
        s = np.ldexp(1.0, np.where(top > 0, np.clip(_floor_log2(top) - 2, -127, 127), -127))
    else:
        most = top.max(axis=1, keepdims=True) if by_row else top.max()
        common = np.ldexp(1.0, np.where(most > 0, np.maximum(_floor_log2(most) - 10, -126), 0))
        s = round_e4m3(top / 6.0 / common) * common
    q = round_e2m1(g / np.where(s > 0, s, 1.0)[:, :, None])
    return np.where(s[:, :, None] > 0, q, 0.0).reshape(n, d), s


def values(x, group: int, by_row: bool) -> np.ndarray:
    q, s = quantise(x, group, by_row)
    return q * np.repeat(s, group, axis=1)


def fp4_values(W_bits: np.ndarray, group: int) -> np.ndarray:
    """What the packed form of bf16 weights stands for, fp64 [V, d]."""
    return values(bf16_decode(W_bits), group, False)


def exit_head_fp4(h_bits, head, tau, group: int) -> dict:
    """As exit_head, with 4-bit weights and activations; also `size` [M], the largest sum of magnitudes behind a row's logits."""
    _, _, y = _rows(h_bits, head)
    y4 = values(bf16_by_f32(y), group, True)
    W4 = fp4_values(head["W"], group)
    out = softmax_stats(y4 @ W4.T)
    tau_arr = np.broadcast_to(np.asarray(tau, dtype=np.float64), (h_bits.shape[0],))
    out["exit_mask"] = exit_decision(out["entropy"], tau_arr)
    out["tau_margin"] = np.abs(out["entropy"] - tau_arr)
    out["size"] = (np.abs(y4) @ np.abs(W4).T).max(axis=1)
    return out
