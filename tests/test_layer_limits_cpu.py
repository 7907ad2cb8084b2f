"""The layer operators' limit on results, at the edge: what is refused as such and
what is taken (and, without a handle, gets as far as the handle)."""
import pytest

from paper_2103_03231_amd import binding as b
from test_layers_abi_cpu import backward, forward, linear, mat, refused


# a launch counts 2^32 - 1 threads: 2^24 - 8 workgroups of 256, a tile of 128 x 128
# each; their number is rounded up to a multiple of eight
@pytest.mark.parametrize("tiles_m,tiles_n,taken", [
    ((1 << 24) - 8, 1, True), (((1 << 24) - 16) // 3, 3, True), (65281, 257, False), (65280, 257, True), (((1 << 24) - 1) // 3, 3, False),
    # up to 256 columns tiles are not workgroups
    ((1 << 24) - 1, 1, True), (1 << 24, 1, False), ((1 << 23) - 1, 2, True)])
def test_results_of_a_launch(tiles_m, tiles_n, taken):
    rows, cols = tiles_m * 128 - 1, tiles_n * 128
    assert rows * cols < 1 << 38
    x = mat(b.MXFP4, rows, 8)
    for call in (linear(rows=rows, n_in=8, n_out=cols, x=x, ws=None, ws_bytes=0), forward(rows=rows, n_in=8, n_out=cols), backward(rows=rows, n_in=8, n_out=cols),
                 backward(rows=rows, n_in=cols, n_out=8)):
        if taken:
            refused(call, "handle is NULL")
        else:
            refused(call, "more results", b.E_UNSUPPORTED)
