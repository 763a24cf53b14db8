"""What the loss's passes ask for: pieces of the vocabulary, not the whole of it."""
import pytest

import paper_2312_06881_amd as dy

MB = 2 ** 20
SIZES = [(129, 4096, 128256), (512, 4096, 50000), (512, 4100, 50000), (4096, 4096, 32768), (1024, 16384, 128256), (64, 768, 2 ** 22),
         (16384, 768, 50000), (300, 1000, 777)]


@pytest.mark.parametrize("dtype", [dy.F32, dy.BF16])
@pytest.mark.parametrize("M,n,V", SIZES)
def test_workspaces_do_not_grow_with_the_vocabulary(M, n, V, dtype):
    if dtype == dy.F32 and M < 129:
        pytest.skip("no weights are laid out")
    value = 6 if dtype == dy.F32 else 2
    # a piece of W laid out otherwise: 768 MB, or the columns of one tile of 256 on each of 256 CUs
    np = -(-n // 64) * 64
    weights = max(768 * MB, (65536 // -(-M // 256) + 512) * np * value)
    # X, X times dloss and the tokens' places, rows padded to 64; by them their tiles' statistics
    rows = M * (n + 64) * (value + 2) + 64 * (M + 512)
    forward = dy.dyad_linear_ce_workspace_bytes(dy.CE_FORWARD, M, n, V, dtype)
    assert 0 < forward <= weights + rows + 8 * M * (V // 128 + 1) + MB
    # G: 512 MB, and 1 / 64 of it for its rows' largest values.  dX's sums: 256 MB over those of one split.
    backward = dy.dyad_linear_ce_workspace_bytes(dy.CE_BACKWARD, M, n, V, dtype)
    assert 0 < backward <= weights + (512 + 8 + 256) * MB + rows + 4 * (M + 64) * n + 16 * n + MB
    # one copy of W at a time, for its logits or turned round
    assert backward <= V * np * value + (512 + 8 + 256) * MB + rows + 4 * (M + 64) * n + 512 * np * value + 16 * n + MB


def test_pieces_of_very_long_rows_are_not_shorter_than_2048_columns():
    n = 2 ** 20
    assert dy.dyad_linear_ce_workspace_bytes(dy.CE_BACKWARD, 64, n, 2048, dy.BF16) >= 2 * 2048 * n
