"""The workspace of the 4-bit floating-point heads for one number of rows is enough for fewer: host-only, nothing touches a device."""
import pytest

from test_abi import lib  # noqa: F401  (the library, built if need be)


@pytest.mark.parametrize("d,V,group", [(1024, 50304, 16), (2560, 50304, 32), (32, 1, 16), (96, 130, 32), (8192, 1000, 16), (64, 1 << 30, 16)])
def test_a_workspace_for_more_rows_serves_fewer(lib, d, V, group):  # noqa: F811
    """A decoding loop allocates for its largest batch.  With 257 rows instead of 256 the states of fewer CTAs meet in a row, 1.4 MB instead of 2.3."""
    f, last = lib.ee_exit_head_fp4_workspace_bytes, 0
    for M in [*range(0, 2100), *range(2100, 40000, 61), *range(40000, 1 << 30, 7654321), 1 << 30]:
        now = f(M, d, V, group)
        assert now >= last > 0 or M == 0, (M, now, last)
        last = now


def test_and_stays_what_the_kernels_need(lib):  # noqa: F811
    """At V = 50304 a row tile of 256 rows is shared by at most 132 of 128 workers' runs of three tiles, four states of 16 bytes each."""
    f = lib.ee_exit_head_fp4_workspace_bytes
    assert f(256, 1024, 50304, 16) >= 256 * 132 * 4 * 16 + 2 * 8 * 9216 + 1024
    assert f(257, 1024, 50304, 16) < f(256, 1024, 50304, 16) + 2 * 8 * 9216 + 100000
