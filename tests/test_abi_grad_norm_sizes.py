"""The gradient norm's workspace at the largest numbers of tensors: host-only, nothing touches a device."""
import ctypes as C

from test_abi import lib  # noqa: F401  (the library, built if need be)


def test_as_many_tensors_as_there_may_be(lib):  # noqa: F811
    """2048 sums of 8 bytes for every 512 tensors; the count was rounded up, and the CTAs numbered, in 32 bits, whatever it was."""
    from paper_2407_21082_b200._lib import EETensor

    f = lib.ee_grad_norm_workspace_bytes
    control = f(1) - 2048 * 8
    for n in (512, 513, 2 ** 29 - 1, 2 ** 29):
        assert f(n) == control + (n + 511) // 512 * 2048 * 8, n
    page, one = C.c_void_p(4096), (EETensor * 1)()
    for n in (2 ** 29 + 1, 2 ** 31 - 512, 2 ** 31 - 1):
        assert f(n) == 0, n
        assert lib.ee_grad_norm(one, n, page, page, 1 << 40, None) == 2 and lib.ee_grad_clip(one, None, n, 1.0, page, None) == 2, n
