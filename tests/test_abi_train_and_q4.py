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
