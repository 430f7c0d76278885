"""Sizes of the cross-entropy's workspaces (host arithmetic, no GPU): they grow with M + V and with what one piece of the logits takes, not
with all M x V of them."""
import pytest

MB = 1 << 20


@pytest.fixture(scope="module")
def ee():
    import paper_2407_21082_b200 as ee
    return ee


def _up(n, k):
    return (n + k - 1) // k * k


@pytest.mark.parametrize("M,d,V", [(1, 8, 1), (64, 512, 50304), (1024, 64, 50304), (1025, 64, 50304), (16384, 2560, 50304), (65536, 1024, 50304),
                                   (131072, 512, 128256)])
def test_the_loss_keeps_two_numbers_per_tile_and_row(ee, M, d, V):
    """Tiles are 256 columns wide from 1025 rows on, at least 64 for fewer."""
    parts = 8 * max(-(-V // 256) * M, -(-V // 64) * min(M, 1024))
    assert ee.ee_head_ce_workspace_bytes(M, d, V) <= M * _up(d, 64) * 2 + parts + 12 * M + 4096


@pytest.mark.parametrize("M,d,V", [(64, 512, 50304), (4096, 1024, 50304), (16384, 2560, 50304), (65536, 1024, 50304), (131072, 512, 128256),
                                   (2 ** 21, 8, 1000)])
def test_the_gradient_keeps_a_piece_of_2_gb_at_most(ee, M, d, V):
    """Beside the loss's: a piece of G (512 MB; up to 2 GB where 74 tiles of dW, 256 rows and up to 256 columns each, take more; 256
    columns where those are more), dy in up to 32 slabs for few rows and one for many, and the strips' column sums."""
    slabs = 32 if M <= 4096 else 1
    piece = max(512 * MB, min(2048 * MB, 512 * M * -(-74 // -(-d // 256))), 512 * M)
    beside = piece + slabs * M * d * 4 + 296 * 8 * 2 * d * 4 + 4096
    assert ee.ee_head_ce_grad_workspace_bytes(M, d, V) <= ee.ee_head_ce_workspace_bytes(M, d, V) + beside
