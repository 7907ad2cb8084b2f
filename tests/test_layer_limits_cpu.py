"""The layer operators' limits: on results, at the edge (what is refused as such, and
what is taken and, without a handle, gets as far as the handle), and on what the
workgroups of a compute unit share, read from the library's code object."""
import re
import struct

import pytest

from paper_2103_03231_amd import binding as b
from test_code_object import LDS_PER_CU, _gfx950_code_objects, _sections
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


# layer_rows_kernel<OP, KS, WN, TA, SRC, EPI, workgroups of a compute unit>
ROWS = re.compile(r"17layer_rows_kernelILi\dELi\dELi\dELb\dELi\dELi\dELi(\d)EEEv")
SIMDS, VGPRS, WAVES = 4, 512, 8        # of a compute unit, of a SIMD's lane, of a workgroup


def test_workgroups_that_a_launch_counts_on_share_a_compute_unit():
    seen = {1: 0, 2: 0}
    for co in _gfx950_code_objects(b.LIB_PATH):
        secs, raw = _sections(co)
        symbols, names = secs[".symtab"], secs[".strtab"]
        for i in range(symbols[5] // 24):
            st_name, _, _, st_shndx, st_value, _ = struct.unpack_from("<IBBHQQ", co, symbols[4] + 24 * i)
            name = co[names[4] + st_name:co.index(b"\0", names[4] + st_name)].decode()
            if not name.endswith(".kd") or "layer_rows_kernel" not in name:
                continue
            kd = co[raw[st_shndx][4] + (st_value - raw[st_shndx][3]):][:64]
            lds, = struct.unpack_from("<I", kd, 0)
            vgprs = 8 * ((struct.unpack_from("<I", kd, 48)[0] & 63) + 1)      # accumulators among them
            count = int(ROWS.search(name).group(1))
            assert count * lds <= LDS_PER_CU and count * WAVES * vgprs <= SIMDS * VGPRS, (name, lds, vgprs)
            seen[count] += 1
    assert seen[1] > 0 and seen[2] > 0, seen
