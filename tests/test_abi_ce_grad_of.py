"""Argument checks of ee_head_ce_grad_of: those of ee_head_ce_grad, with ce before lse (host-only, nothing touches a device)."""
import ctypes

from test_abi import lib  # noqa: F401  (the library, built if need be)


def test_argument_errors(lib):
    N, p, off = None, ctypes.c_void_p(4096), ctypes.c_void_p(4104)      # never read: the checks come first
    tail = (p, 1 << 30, N)
    for ce in (N, p):
        def call(lse=p, loss=p, dce=N, dloss=N, ld_dh=64, dW=p, dbeta=p, end=tail):
            return lib.ee_head_ce_grad_of(p, 64, p, p, 1e-5, p, 4, 64, 100, p, ce, lse, loss, dce, dloss, p, ld_dh, dW, p, dbeta, 0, *end)
        assert call(dce=p, dloss=p) == 2 and call(dbeta=N) == 1 and call(ld_dh=60) == 2 and call(dW=off) == 3
        assert call(lse=N) == 1 and call(loss=N) == 1 and call(end=(p, 256, N)) == 4
        assert lib.ee_head_ce_grad_of(p, 64, p, p, 1e-5, p, 4, 64, 100, p, ce, p, p, N, N, N, 0, N, N, N, 0, *tail) == 0      # nothing asked for
    assert lib.ee_head_ce_grad_of(p, 64, p, p, 1e-5, p, 4, 60, 100, p, p, p, p, N, N, p, 64, p, p, p, 0, *tail) == 2
