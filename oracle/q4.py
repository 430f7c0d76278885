"""fp64 CPU oracle for heads held in 4 bits (see include/eexit.h, "Heads held in 4 bits") and for the embedding.

TEST INFRASTRUCTURE ONLY (see oracle/exit_head.py).  Shares no code with the CUDA sources.
"""
from __future__ import annotations

import numpy as np

from .exit_head import bf16_decode, bf16_rne


def q4_quantise(W_bits: np.ndarray, group: int):
    """Whole numbers [V, d] and scales [V, d / group] of bf16 weights."""
    W = bf16_decode(W_bits)
    V, d = W.shape
    w = W.reshape(V, d // group, group)
    # max / 7 has no finite binary expansion unless it is exact, so rounding it to fp32 first cannot land on a bf16 midpoint
    s = bf16_rne((np.abs(w).max(axis=2) / 7.0).astype(np.float32).astype(np.float64))
    safe = np.where(s > 0, s, 1.0)[:, :, None]
    q = np.clip(np.rint(w / safe), -8, 7)
    return np.where(s[:, :, None] > 0, q, 0.0).reshape(V, d), s


def q4_values(W_bits: np.ndarray, group: int) -> np.ndarray:
    """bf16 bit patterns of what the 4-bit form stands for."""
    q, s = q4_quantise(W_bits, group)
    v = bf16_rne(q * np.repeat(s, group, axis=1))
    return (v.astype(np.float32).view(np.uint32) >> np.uint32(16)).astype(np.uint16)


def embed(table_bits, tokens, scale) -> np.ndarray:
    table = bf16_decode(table_bits)
    ok = (tokens >= 0) & (tokens < table.shape[0])
    return np.where(ok[:, None], table[np.where(ok, tokens, 0)] * float(scale), 0.0)


def embed_grad(dout_bits, tokens, V, scale):
    """The gradient [V, d], and per element the sum of magnitudes and per row the number of terms."""
    dout = bf16_decode(dout_bits)
    ok = (tokens >= 0) & (tokens < V)
    out, size = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1]))
    np.add.at(out, tokens[ok], dout[ok] * float(scale))
    np.add.at(size, tokens[ok], np.abs(dout[ok] * float(scale)))
    return out, size, np.bincount(tokens[ok], minlength=V)
