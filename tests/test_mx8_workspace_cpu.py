"""Workspaces of the passes over int8 checkpoints: none where an epilogue keeps and reads the 8 bits."""
import pytest

import paper_2312_06881_amd as dy

VARIANTS = (dy.IT, dy.OT, dy.DT)


def need(pass_, variant, n_in, n_out, D, M, dtype=dy.BF16):
    return dy.dyad_mx8_workspace_bytes(pass_, variant, n_in, n_out, D, M, dtype, dy.ACT_NONE)


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("shape", [(768, 3072, 4, 16384), (3072, 768, 4, 1), (1024, 4096, 4, 257), (2048, 8192, 8, 5000),
                                   (256, 512, 1, 100), (512, 1024, 2, 64)], ids=lambda s: "x".join(map(str, s)))
def test_no_copy_where_the_epilogue_does_it(shape, variant):
    n_in, n_out, D, M = shape
    assert need(dy.MX8_FORWARD, variant, n_in, n_out, D, M) == 0
    assert need(dy.MX8_DX, variant, n_in, n_out, D, M) == 0
    # the weight gradient reads a copy of the layer's input
    assert need(dy.MX8_DW, variant, n_in, n_out, D, M) >= 2 * M * n_in


@pytest.mark.parametrize("variant", VARIANTS)
def test_a_copy_where_none_does(variant):
    for shape, dtype in (((768, 3072, 4, 600), dy.F32), ((770, 615, 5, 600), dy.BF16), ((768, 3072, 5, 600), dy.BF16),
                         ((64, 256, 4, 8), dy.BF16), ((896, 896, 7, 300), dy.BF16)):
        n_in, n_out, D, M = shape
        size = 2 if dtype == dy.BF16 else 4
        assert need(dy.MX8_FORWARD, variant, *shape, dtype) == (M * n_out * size + 255) // 256 * 256
        assert need(dy.MX8_DX, variant, *shape, dtype) == (M * n_in * size + 255) // 256 * 256


def test_copies_are_bounded():
    """Of a long batch a part is copied at a time."""
    assert need(dy.MX8_FORWARD, dy.IT, 768, 3072, 5, 1 << 20) <= 64 << 20
    assert need(dy.MX8_DX, dy.IT, 1 << 20, 5, 5, 4096, dy.F32) == 1024 * 4 << 20
    for variant in VARIANTS:
        for pass_ in (dy.MX8_FORWARD, dy.MX8_DX):
            assert need(pass_, variant, 768, 3072, 5, 0) == 0


def test_columns_that_only_buffered_kernels_take_keep_their_copy():
    """n_dyad 6 under an output transpose sums its components in the stream's buffer, which a stream that
    is being captured may not have: the copy stays for that call."""
    assert need(dy.MX8_FORWARD, dy.IT, 768, 1536, 6, 2050) == 0
    assert need(dy.MX8_FORWARD, dy.OT, 768, 1536, 6, 2050) > 0
    assert need(dy.MX8_DX, dy.IT, 768, 1536, 6, 2050) > 0
    assert need(dy.MX8_DX, dy.OT, 768, 1536, 6, 2050) == 0
