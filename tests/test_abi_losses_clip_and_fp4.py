"""Argument checks of the token losses, the gradient norm and the 4-bit floating-point heads: host-only, nothing touches a device."""
import ctypes as C

from test_abi import lib  # noqa: F401  (the library, built if need be)

N, P, OFF, BIG = None, C.c_void_p(4096), C.c_void_p(4104), 1 << 40
OVER = (1 << 30) + 1


def test_argument_errors_of_the_policy_loss(lib):
    nan, inf = float("nan"), float("inf")

    def call(ce=P, old=P, ref=P, adv=P, labels=P, M=4, V=10, starts=N, S=0, counted=P, low=0.2, high=0.2, kl=0.1, dce=P, loss=P, ws=P, n=BIG):
        return lib.ee_policy_loss(ce, old, ref, adv, labels, M, V, starts, S, counted, low, high, kl, dce, loss, ws, n, N)

    for bad in (dict(M=-1), dict(M=OVER), dict(V=0), dict(V=OVER), dict(starts=P, S=0), dict(starts=P, S=OVER), dict(low=-0.1), dict(low=1.1), dict(low=nan),
                dict(high=-0.1), dict(high=nan), dict(kl=-1.0), dict(kl=nan), dict(ref=N)):
        assert call(**bad) == 2, bad
    for bad in (dict(ce=N), dict(old=N), dict(adv=N), dict(labels=N), dict(counted=N), dict(dce=N), dict(loss=N), dict(ws=N), dict(starts=P, S=2, adv=N)):
        assert call(**bad) == 1, bad
    assert call(ws=OFF) == 3 and call(n=lib.ee_token_loss_workspace_bytes() - 1) == 4
    assert call(high=inf, n=1) == 4                                      # an open clip is allowed
    assert lib.ee_token_loss_workspace_bytes() % 256 == 0


def test_argument_errors_of_the_preference_loss(lib):
    def call(ce=P, ref=N, labels=P, M=4, V=10, starts=P, pairs=2, beta=0.1, soft=0.0, dce=P, margin=P, loss=P, ws=P, n=BIG):
        return lib.ee_preference_loss(ce, ref, labels, M, V, starts, pairs, beta, soft, dce, margin, loss, ws, n, N)

    for bad in (dict(M=-1), dict(V=0), dict(pairs=0), dict(pairs=OVER), dict(beta=-1.0), dict(beta=float("nan")), dict(soft=1.5), dict(soft=-0.5)):
        assert call(**bad) == 2, bad
    for bad in (dict(ce=N), dict(labels=N), dict(starts=N), dict(dce=N), dict(margin=N), dict(loss=N), dict(ws=N)):
        assert call(**bad) == 1, bad
    assert call(ws=OFF) == 3 and call(n=4096) == 4


def test_argument_errors_of_the_gradient_norm(lib):
    from paper_2407_21082_b200._lib import EETensor

    def tensors(*rows):
        arr = (EETensor * max(1, len(rows)))()
        for t, (data, n, kind) in zip(arr, rows):
            t.data, t.n, t.type = data, n, kind
        return arr

    def norm(rows, count=None, out=P, ws=P, n=BIG):
        return lib.ee_grad_norm(tensors(*rows), len(rows) if count is None else count, out, ws, n, N)

    good = (4096, 10, 0)
    assert norm([good], count=-1) == 2 and norm([(4096, -1, 0)]) == 2 and norm([(4096, 10, 3)]) == 2 and norm([(4096, (1 << 36) + 1, 0)]) == 2
    assert norm([(4096, 1 << 36, 0)] * 200) == 2                         # together beyond what is numbered
    assert norm([good, (None, 10, 0)]) == 1 and norm([good], out=N) == 1 and norm([good], ws=N) == 1
    assert lib.ee_grad_norm(N, 1, P, P, BIG, N) == 1
    assert norm([(4097, 10, 0)]) == 3 and norm([(4098, 10, 2)]) == 3 and norm([good], ws=OFF) == 3
    assert norm([good], n=lib.ee_grad_norm_workspace_bytes(1) - 1) == 4
    f = lib.ee_grad_norm_workspace_bytes
    assert f(-1) == 0 and f(0) == f(512) and f(513) > f(512)

    def clip(rows, out=None, max_norm=1.0, value=P):
        arr = None if out is None else (C.c_void_p * len(out))(*out)
        return lib.ee_grad_clip(tensors(*rows), arr, len(rows), max_norm, value, N)

    assert clip([good], max_norm=-1.0) == 2 and clip([good], max_norm=float("nan")) == 2 and clip([good], value=N) == 1
    assert clip([good], out=[None]) == 1 and clip([good], out=[4097]) == 3 and clip([(4096, 10, 2)], out=[4098]) == 3


def test_argument_errors_of_the_4_bit_floating_point_heads(lib):
    f, g = lib.ee_head_fp4_bytes, lib.ee_exit_head_fp4_workspace_bytes
    for bad in [(0, 64, 16), (5, 64, 8), (5, 40, 16), (5, 48, 32), (5, 8208, 16), (5, 64, 64), (-1, 64, 16), (OVER, 64, 16)]:
        assert f(*bad) == 0 and g(4, bad[1], bad[0], bad[2]) == 0
    # half a byte per weight and one per group, in units of 128 by 128
    assert f(128, 128, 16) == 256 + 8192 + 1024 and f(128, 128, 32) == 256 + 8192 + 512
    assert f(50304, 1024, 16) == 256 + 393 * 8 * 9216 and f(1 << 30, 16, 16) == 256 + (1 << 23) * 9216
    assert g(-1, 64, 10, 16) == 0 and g(OVER, 64, 10, 16) == 0 and g(0, 64, 10, 16) >= 256 and g(1 << 30, 64, 10, 32) > 0
    assert lib.ee_head_fp4_pack(P, 5, 40, 16, P, BIG, N) == 2 and lib.ee_head_fp4_pack(N, 5, 64, 16, P, BIG, N) == 1
    assert lib.ee_head_fp4_unpack(P, BIG, 5, 64, 16, N, N) == 1
    assert lib.ee_head_fp4_pack(OFF, 5, 64, 16, P, BIG, N) == 3 and lib.ee_head_fp4_pack(P, 5, 64, 16, OFF, BIG, N) == 3
    assert lib.ee_head_fp4_pack(P, 5, 64, 16, P, 512, N) == 4 and lib.ee_head_fp4_unpack(P, 512, 5, 64, 16, P, N) == 4
    ok = (P, P, P, P, P, BIG, N)
    assert lib.ee_exit_head_fp4(P, 64, P, P, 1e-5, P, BIG, 48, 4, 64, 10, N, 1.0, *ok) == 2
    assert lib.ee_exit_head_fp4(P, 56, P, P, 1e-5, P, BIG, 16, 4, 64, 10, N, 1.0, *ok) == 2
    assert lib.ee_exit_head_fp4(P, 64, P, P, 1e-5, P, BIG, 16, OVER, 64, 10, N, 1.0, *ok) == 2
    assert lib.ee_exit_head_fp4(P, 64, P, P, 1e-5, N, BIG, 16, 4, 64, 10, N, 1.0, *ok) == 1
    assert lib.ee_exit_head_fp4(P, 64, P, P, 1e-5, OFF, BIG, 16, 4, 64, 10, N, 1.0, *ok) == 3
    assert lib.ee_exit_head_fp4(P, 64, P, P, 1e-5, P, 64, 16, 4, 64, 10, N, 1.0, *ok) == 4
    assert lib.ee_exit_head_fp4(P, 64, P, P, 1e-5, P, BIG, 16, 4, 64, 10, N, 1.0, P, P, P, P, P, 256, N) == 4
    assert lib.ee_exit_head_fp4(N, 64, N, N, 1e-5, N, 0, 16, 0, 64, 10, N, 1.0, N, N, N, N, N, 0, N) == 0
