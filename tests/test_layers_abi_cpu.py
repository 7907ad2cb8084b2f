"""What the layer operators refuse, through the C ABI and without a GPU: every
argument is checked before the handle and any HIP call, so calls without a
handle show each check by its message."""
import pytest

from paper_2103_03231_amd import binding as b

A = 1 << 20       # an aligned address; nothing reads it
F32, BF16 = b.TYPE_FP32, b.TYPE_BF16


def mat(kind, rows, cols, **kw):
    blocks = -(-cols // 32)
    d = {"data": A, "ld": cols if kind in (F32, BF16) else blocks * (16 if kind == b.MXFP4 else 32), "type": kind,
         "scales": None if kind in (F32, BF16) else A, "ld_scales": 0 if kind in (F32, BF16) else -(-blocks // 8) * 8}
    d.update(kw)
    return (d["data"], d["ld"], d["type"], d["scales"], d["ld_scales"])


def refused(call, message, status=b.E_INVALID_ARG):
    with pytest.raises(b.DonerfError) as e:
        call()
    assert e.value.status == status and message in str(e.value), str(e.value)


def quantize(rows=4, cols=100, x=None, q=None):
    return lambda: b.donerf_mx_quantize(None, x if x else mat(F32, rows, cols), q if q else mat(b.MXFP4, rows, cols), rows, cols)


def dequantize(rows=4, cols=100, q=None, y=None):
    return lambda: b.donerf_mx_dequantize(None, q if q else mat(b.MXFP8, rows, cols), y if y else mat(BF16, rows, cols), rows, cols)


def linear(rows=4, n_in=100, n_out=40, x=None, w=None, bias=None, relu=0, y=None, ws=A, ws_bytes=None):
    need = b.donerf_mx_linear_workspace(BF16, rows, n_in)
    return lambda: b.donerf_mx_linear(None, x if x else mat(BF16, rows, n_in), w if w else mat(b.MXFP4, n_out, n_in), bias, relu,
                                      y if y else mat(BF16, rows, n_out), rows, n_in, n_out, ws, need if ws_bytes is None else ws_bytes)


def forward(rows=4, n_in=100, n_out=40, x=None, w=None, bias=None, relu=0, y="y", kept="kept"):
    y = mat(BF16, rows, n_out) if y == "y" else y
    kept = mat(b.MXFP8, rows, n_out) if kept == "kept" else kept
    return lambda: b.donerf_train_linear(None, x if x else mat(BF16, rows, n_in), w if w else mat(BF16, n_out, n_in), bias, relu,
                                         y, kept, rows, n_in, n_out)


def backward(rows=4, n_in=100, n_out=40, dz=None, x=None, relu=0, w="w", dx="dx", dw="dw", db=A, accumulate=0):
    w = mat(BF16, n_out, n_in) if w == "w" else w
    dx = mat(BF16, rows, n_in) if dx == "dx" else dx
    dw = mat(F32, n_out, n_in) if dw == "dw" else dw
    return lambda: b.donerf_train_linear_backward(None, dz if dz else mat(BF16, rows, n_out), x if x else mat(b.MXFP8, rows, n_in), relu,
                                                  w, dx, dw, db, accumulate, rows, n_in, n_out, A, 1 << 40)


@pytest.mark.parametrize("call", [quantize(), dequantize(), linear(), forward(), backward(), forward(y=None), forward(kept=None),
                                  backward(dx=None, w=None), backward(dw=None, db=None), backward(db=None),
                                  linear(x=mat(b.MXFP4, 4, 100), ws=None), linear(rows=0, ws=None), quantize(rows=0),
                                  quantize(rows=0, x=mat(F32, 0, 100, data=None), q=mat(b.MXFP8, 0, 100, data=None, scales=None)),
                                  backward(rows=0), quantize(rows=1, cols=1), quantize(cols=b.MAX_COLS),
                                  quantize(x=mat(BF16, 4, 100, ld=101, data=A + 2)), forward(w=mat(BF16, 40, 100, data=A + 6, ld=333))])
def test_good_arguments_get_as_far_as_the_handle(call):
    refused(call, "handle is NULL")


MATRICES = [
    # (call with the matrix given, its name, its type, rows, cols)
    (lambda m: quantize(x=m), "x", F32, 4, 100), (lambda m: quantize(q=m), "q", b.MXFP4, 4, 100),
    (lambda m: dequantize(q=m), "q", b.MXFP8, 4, 100), (lambda m: dequantize(y=m), "y", F32, 4, 100),
    (lambda m: linear(x=m), "x", BF16, 4, 100), (lambda m: linear(w=m), "w", b.MXFP4, 40, 100), (lambda m: linear(y=m), "y", b.MXFP4, 4, 40),
    (lambda m: forward(x=m), "x", BF16, 4, 100), (lambda m: forward(w=m), "w", BF16, 40, 100), (lambda m: forward(y=m), "y", BF16, 4, 40),
    (lambda m: forward(kept=m), "kept", b.MXFP8, 4, 40),
    (lambda m: backward(dz=m), "dz", BF16, 4, 40), (lambda m: backward(x=m), "x", b.MXFP8, 4, 100), (lambda m: backward(x=m), "x", BF16, 4, 100),
    (lambda m: backward(w=m), "w", BF16, 40, 100), (lambda m: backward(dx=m), "dx", BF16, 4, 100), (lambda m: backward(dw=m), "dw", F32, 40, 100),
]


@pytest.mark.parametrize("call,name,kind,rows,cols", MATRICES)
def test_bad_matrices(call, name, kind, rows, cols):
    good = mat(kind, rows, cols)
    refused(call(good), "handle is NULL")
    step = {F32: 4, BF16: 2}.get(kind, 16)
    bad = [({"data": None}, "NULL buffer"), ({"data": A + step // 2}, "not aligned"), ({"ld": good[1] - 1}, "ld out of range"),
           ({"ld": 0}, "ld out of range"), ({"ld": -good[1]}, "ld out of range"), ({"ld": 1 << 41}, "ld out of range"),
           ({"type": 4}, "type is not taken"), ({"type": -1}, "type is not taken"), ({"type": 40}, "type is not taken")]
    if kind in (F32, BF16):
        bad += [({"scales": A}, "scales given")]
    else:
        bad += [({"scales": None}, "NULL buffer"), ({"scales": A + 4}, "not aligned"), ({"ld": good[1] + 8}, "multiple of 16"),
                ({"ld_scales": 4}, "multiple of 8"), ({"ld_scales": 0}, "multiple of 8"), ({"ld_scales": 12}, "multiple of 8")]
    for kw, message in bad:
        refused(call(mat(kind, rows, cols, **kw)), f"{name}: ")
        refused(call(mat(kind, rows, cols, **kw)), message)


@pytest.mark.parametrize("call,kinds", [
    (lambda m: quantize(x=m), (b.MXFP4, b.MXFP8)), (lambda m: quantize(q=m), (F32, BF16)), (lambda m: dequantize(y=m), (b.MXFP4, b.MXFP8)),
    (lambda m: linear(x=m), (b.MXFP8,)), (lambda m: linear(w=m), (F32, BF16, b.MXFP8)), (lambda m: linear(y=m), (b.MXFP8,)),
    (lambda m: forward(x=m), (F32, b.MXFP4, b.MXFP8)), (lambda m: forward(kept=m), (F32, BF16, b.MXFP4)),
    (lambda m: backward(dz=m), (F32, b.MXFP8)), (lambda m: backward(x=m), (F32, b.MXFP4)), (lambda m: backward(dw=m), (BF16,)),
])
def test_types_that_are_not_taken(call, kinds):
    for kind in kinds:
        refused(call(mat(kind, 100, 100)), "type is not taken")


def test_missing_matrices():
    refused(lambda: b.donerf_mx_quantize(None, None, mat(b.MXFP4, 1, 8), 1, 8), "x: NULL")
    refused(lambda: b.donerf_mx_linear(None, mat(BF16, 1, 8), None, None, 0, mat(BF16, 1, 8), 1, 8, 8), "w: NULL")
    refused(forward(y=None, kept=None), "neither y nor kept")
    refused(backward(w=None), "w: NULL")
    refused(backward(dx=None, dw=None, db=None), "no gradient")


@pytest.mark.parametrize("make", [quantize, dequantize])
def test_sizes_of_conversions(make):
    for rows, cols in ((-1, 8), (1 << 31, 8), (4, 0), (4, -3), (4, b.MAX_COLS + 1)):
        refused(make(rows=rows, cols=cols, **({"x": mat(F32, 1, 8), "q": mat(b.MXFP4, 1, 8)} if make is quantize else
                                              {"q": mat(b.MXFP4, 1, 8), "y": mat(F32, 1, 8)})), "must lie in")


@pytest.mark.parametrize("make", [linear, forward, backward])
def test_sizes_of_layers(make):
    for rows, n_in, n_out in ((-1, 8, 8), (1 << 31, 8, 8), (4, 0, 8), (4, 8, 0), (4, b.MAX_COLS + 1, 8), (4, 8, b.MAX_COLS + 1)):
        refused(make(rows=rows, n_in=n_in, n_out=n_out), "must lie in")
    # results that a launch's grid cannot count
    for wide in ({"n_in": b.MAX_COLS}, {"n_out": b.MAX_COLS}) if make is backward else ({"n_out": b.MAX_COLS},):
        refused(make(rows=(1 << 31) - 1, **wide), "more results", b.E_UNSUPPORTED)


def test_offsets_that_64_bits_would_not_hold():
    rows = (1 << 31) - 1
    refused(quantize(rows=rows, cols=8, x=mat(F32, rows, 8, ld=1 << 40)), "x: ld out of range")
    refused(quantize(rows=rows, cols=8, q=mat(b.MXFP4, rows, 8, ld_scales=1 << 40)), "q: ld_scales")
    refused(quantize(rows=rows, cols=8), "handle is NULL")


def test_flags_bias_and_workspace():
    for make in (linear, forward):
        refused(make(relu=2), "relu must be")
        refused(make(bias=A + 2), "bias not aligned")
        refused(make(bias=A), "handle is NULL")
    refused(backward(relu=-1), "must be 0 or 1")
    refused(backward(accumulate=2), "must be 0 or 1")
    refused(backward(db=A + 1), "db not aligned")
    need = b.donerf_mx_linear_workspace(BF16, 100, 100)
    assert need == 100 * 64 + 100 * 8
    refused(linear(rows=100, ws_bytes=need - 1), "workspace of", b.E_SIZE)
    refused(linear(rows=100, ws=None), "workspace is NULL")
    refused(linear(rows=100, ws=A + 8), "workspace not aligned")
    # a few rows need none
    assert b.donerf_mx_linear_workspace(BF16, 32, 100) == 0 < b.donerf_mx_linear_workspace(BF16, 33, 100)
    refused(linear(rows=32, ws=None), "handle is NULL")
    assert b.donerf_mx_linear_workspace(b.MXFP4, 4, 100) == 0 == b.donerf_mx_linear_workspace(F32, -1, 100)
    assert b.donerf_mx_linear_workspace(F32, 4, 0) == 0 == b.donerf_mx_linear_workspace(F32, 4, b.MAX_COLS + 1)
    assert b.donerf_train_linear_backward_workspace(None, 4, 4, 4) == 0


def test_get_stream_without_a_handle():
    refused(lambda: b.donerf_get_stream(None), "handle is NULL")
