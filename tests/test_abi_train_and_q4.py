"""Argument checks of the training, 4-bit and embedding entry points: host-only, nothing touches a device."""
import ctypes

from test_abi import lib  # noqa: F401  (the library, built if need be)


def test_argument_errors_of_the_cross_entropy(lib):
    """ee_head_ce and ee_head_ce_grad: sizes and validation, before any launch."""
    N = None
    f, g = lib.ee_head_ce_workspace_bytes, lib.ee_head_ce_grad_workspace_bytes
    for bad in [(-1, 512, 10), (8, 513, 10), (8, 4, 10), (8, 512, 0), (8, 8200, 10)]:
        assert f(*bad) == 0 and g(*bad) == 0
    assert g(4096, 1024, 50304) > f(4096, 1024, 50304) > 4096 * 1024 * 2
    assert g(16384, 2560, 50304) < 16384 * 50304 * 2                     # less than the logits in 16 bits
    assert lib.ee_head_ce(N, 64, N, N, 1e-5, N, 4, 64, 100, N, N, N, N, N, 0, N) == 1
    assert lib.ee_head_ce(N, 64, N, N, 1e-5, N, 4, 60, 100, N, N, N, N, N, 0, N) == 2
    p = ctypes.c_void_p(4096)                                            # never read: the checks come first
    off = ctypes.c_void_p(4104)
    assert lib.ee_head_ce(p, 60, p, p, 1e-5, p, 4, 64, 100, p, p, p, p, p, 1 << 30, N) == 2              # ld_h < d
    assert lib.ee_head_ce(off, 64, p, p, 1e-5, p, 4, 64, 100, p, p, p, p, p, 1 << 30, N) == 3
    assert lib.ee_head_ce(p, 64, p, p, 1e-5, p, 4, 64, 100, p, p, p, p, p, 256, N) == 4
    tail = (p, 1 << 30, N)
    assert lib.ee_head_ce_grad(p, 64, p, p, 1e-5, p, 4, 64, 100, p, p, p, p, p, p, 64, p, p, p, 0, *tail) == 2     # dce and dloss
    assert lib.ee_head_ce_grad(p, 64, p, p, 1e-5, p, 4, 64, 100, p, p, p, N, N, p, 64, p, p, N, 0, *tail) == 1     # dgamma alone
    assert lib.ee_head_ce_grad(p, 64, p, p, 1e-5, p, 4, 64, 100, p, p, p, N, N, p, 60, p, p, p, 0, *tail) == 2     # ld_dh < d
    assert lib.ee_head_ce_grad(p, 64, p, p, 1e-5, p, 4, 64, 100, p, p, p, N, N, p, 64, off, p, p, 0, *tail) == 3
    assert lib.ee_head_ce_grad(p, 64, p, p, 1e-5, p, 4, 64, 100, p, p, N, N, N, p, 64, p, p, p, 0, *tail) == 1     # no loss
    assert lib.ee_head_ce_grad(p, 64, p, p, 1e-5, p, 4, 64, 100, p, p, p, N, N, p, 64, p, p, p, 0, p, 256, N) == 4
    assert lib.ee_head_ce_grad(p, 64, p, p, 1e-5, p, 4, 64, 100, p, p, p, N, N, N, 0, N, N, N, 0, *tail) == 0      # nothing asked for


def test_argument_errors_of_the_4_bit_heads(lib):
    N, p, off = None, ctypes.c_void_p(4096), ctypes.c_void_p(4104)
    f = lib.ee_head_q4_bytes
    for bad in [(0, 64, 64), (5, 64, 16), (5, 96, 64), (5, 32, 64), (5, 8256, 64), (5, 64, 256), (-1, 64, 64)]:
        assert f(*bad) == 0
    # half a byte per weight and two per group, rounded up to tiles
    assert f(16, 64, 64) == 512 + 256 and f(50304, 1024, 64) == 50304 * 512 + 50304 * 16 * 2
    assert lib.ee_head_q4_pack(p, 5, 96, 64, p, 1 << 20, N) == 2 and lib.ee_head_q4_pack(N, 5, 64, 64, p, 1 << 20, N) == 1
    assert lib.ee_head_q4_pack(ctypes.c_void_p(4112), 5, 64, 64, p, 1 << 20, N) == 3                     # 32 bytes, not 16
    assert lib.ee_head_q4_unpack(p, 1 << 20, 5, 64, 64, ctypes.c_void_p(4112), N) == 3
    assert lib.ee_head_q4_pack(off, 5, 64, 64, p, 1 << 20, N) == 3 and lib.ee_head_q4_pack(p, 5, 64, 64, off, 1 << 20, N) == 3
    assert lib.ee_head_q4_pack(p, 5, 64, 64, p, 512, N) == 4 and lib.ee_head_q4_unpack(p, 512, 5, 64, 64, p, N) == 4
    assert lib.ee_head_q4_unpack(p, 1 << 20, 5, 64, 64, N, N) == 1
    assert lib.ee_exit_head_q4_workspace_bytes(8, 60, 10) == 0 and lib.ee_exit_head_q4_workspace_bytes(0, 64, 10) >= 256
    big = 1 << 30
    ok = (p, p, p, p, p, big, N)
    assert lib.ee_exit_head_q4(p, 64, p, p, 1e-5, p, big, 48, 4, 64, 10, N, 1.0, *ok) == 2
    assert lib.ee_exit_head_q4(p, 56, p, p, 1e-5, p, big, 64, 4, 64, 10, N, 1.0, *ok) == 2
    assert lib.ee_exit_head_q4(p, 64, p, p, 1e-5, N, big, 64, 4, 64, 10, N, 1.0, *ok) == 1
    assert lib.ee_exit_head_q4(p, 64, p, p, 1e-5, off, big, 64, 4, 64, 10, N, 1.0, *ok) == 3
    assert lib.ee_exit_head_q4(p, 64, p, p, 1e-5, p, 64, 64, 4, 64, 10, N, 1.0, *ok) == 4
    assert lib.ee_exit_head_q4(p, 64, p, p, 1e-5, p, big, 64, 4, 64, 10, N, 1.0, p, p, p, p, p, 256, N) == 4
    assert lib.ee_exit_head_q4(N, 64, N, N, 1e-5, N, 0, 64, 0, 64, 10, N, 1.0, N, N, N, N, N, 0, N) == 0


def test_argument_errors_of_the_embedding(lib):
    N, p, off = None, ctypes.c_void_p(4096), ctypes.c_void_p(4104)
    assert lib.ee_embed(p, 5, 12, p, 3, 1.0, p, 16, N) == 2 and lib.ee_embed(p, 5, 16, p, 3, 1.0, p, 8, N) == 2
    assert lib.ee_embed(p, 0, 16, p, 3, 1.0, p, 16, N) == 2 and lib.ee_embed(p, 5, 16, p, -1, 1.0, p, 16, N) == 2
    assert lib.ee_embed(N, 5, 16, p, 3, 1.0, p, 16, N) == 1 and lib.ee_embed(off, 5, 16, p, 3, 1.0, p, 16, N) == 3
    assert lib.ee_embed(N, 5, 16, N, 0, 1.0, N, 16, N) == 0
    f = lib.ee_embed_grad_workspace_bytes
    assert f(-1, 16, 5) == 0 and f(4, 12, 5) == 0 and f(4, 16, 0) == 0 and f(0, 16, 5) >= 256
    assert f(16384, 1024, 50304) >= 16384 * 8 and f(16385, 1024, 50304) >= 16385 * 16
    big = 1 << 30
    assert lib.ee_embed_grad(p, 16, p, 3, 5, 12, 1.0, p, 0, 0, p, big, N) == 2
    assert lib.ee_embed_grad(p, 8, p, 3, 5, 16, 1.0, p, 0, 0, p, big, N) == 2
    assert lib.ee_embed_grad(p, 16, p, 3, 5, 16, 1.0, N, 0, 0, p, big, N) == 1
    assert lib.ee_embed_grad(p, 16, p, 3, 5, 16, 1.0, off, 0, 0, p, big, N) == 3
    assert lib.ee_embed_grad(p, 16, p, 3, 5, 16, 1.0, p, 0, 0, p, 64, N) == 4


def test_rows_and_vocabularies_beyond_32_bits_of_tiles_are_refused(lib):
    N, p, big, over = None, ctypes.c_void_p(4096), 1 << 40, (1 << 30) + 1
    for f in (lib.ee_head_ce_workspace_bytes, lib.ee_head_ce_grad_workspace_bytes, lib.ee_exit_head_q4_workspace_bytes, lib.ee_embed_grad_workspace_bytes):
        assert f(over, 8, 10) == 0 and f(1, 8, over) == 0 and f(1, 8, 2 ** 31 - 1) == 0 and f(1, 8, 1 << 30) > 0
    assert lib.ee_head_q4_bytes(over, 32, 32) == 0 and lib.ee_head_q4_bytes(1 << 30, 32, 32) == (1 << 26) * (512 + 2 * 32)          # 64 columns, two groups
    for M, V in [(over, 10), (4, over), (4, 2 ** 31 - 1)]:
        assert lib.ee_head_ce(p, 8, p, p, 1e-5, p, M, 8, V, p, p, p, p, p, big, N) == 2
        assert lib.ee_head_ce_grad(p, 8, p, p, 1e-5, p, M, 8, V, p, p, p, N, N, p, 8, p, p, p, 0, p, big, N) == 2
        assert lib.ee_exit_head_q4(p, 32, p, p, 1e-5, p, big, 32, M, 32, V, N, 1.0, p, p, p, p, p, big, N) == 2
        assert lib.ee_embed(p, V, 8, p, M, 1.0, p, 8, N) == 2
        assert lib.ee_embed_grad(p, 8, p, M, V, 8, 1.0, p, 0, 0, p, big, N) == 2
    assert lib.ee_head_q4_pack(p, over, 32, 32, p, big, N) == 2 and lib.ee_head_q4_unpack(p, big, over, 32, 32, p, N) == 2
