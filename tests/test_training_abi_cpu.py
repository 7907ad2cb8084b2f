"""What the operators around the layers refuse, through the C ABI and without a GPU:
every argument is checked before the handle and any HIP call, so calls without a
handle show each check by its message."""
import math

import pytest

from paper_2103_03231_amd import binding as b
from test_layers_abi_cpu import A, BF16, F32, mat, refused

I32, I64 = b.TYPE_INT32, b.TYPE_INT64


def ints(kind, rows, cols, **kw):
    d = {"data": A, "ld": cols, "type": kind, "scales": None, "ld_scales": 0} | kw
    return (d["data"], d["ld"], d["type"], d["scales"], d["ld_scales"])


def norm(rows=4, cols=100, x=None, weight=A, bias=A, eps=1e-5, relu=0, y="y", kept="kept", stats=A):
    y = mat(BF16, rows, cols) if y == "y" else y
    kept = mat(b.MXFP8, rows, cols) if kept == "kept" else kept
    return lambda: b.donerf_train_norm(None, x if x else mat(F32, rows, cols), weight, bias, eps, relu, y, kept, stats, rows, cols)


def norm_backward(rows=4, cols=100, dz=None, x=None, relu=0, weight=A, stats=A, dx="dx", dw=A, db=A, accumulate=0):
    dx = mat(BF16, rows, cols) if dx == "dx" else dx
    return lambda: b.donerf_train_norm_backward(None, dz if dz else mat(BF16, rows, cols), x if x else mat(b.MXFP8, rows, cols), relu, weight,
                                                stats, dx, dw, db, accumulate, rows, cols, A, 1 << 40)


def lookup(rows=4, n=7, cols=100, table=None, ids=None, scale=1.0, y=None):
    return lambda: b.donerf_train_embedding(None, table if table else mat(BF16, n, cols), ids if ids else ints(I64, rows, 1), scale,
                                            y if y else mat(F32, rows, cols), rows, n, cols)


def lookup_backward(rows=4, n=7, cols=100, dy=None, ids=None, dtable=None, accumulate=0, ws=A, ws_bytes=1 << 50):
    return lambda: b.donerf_train_embedding_backward(None, dy if dy else mat(BF16, rows, cols), ids if ids else ints(I32, rows, 1), 1.0,
                                                     dtable if dtable else mat(F32, n, cols), accumulate, rows, n, cols, ws, ws_bytes)


def distill(rows=4, cols=100, k=3, x=None, classes=None, teacher=None, weight=A, temperature=1.0, loss=A, dx="dx"):
    dx = mat(BF16, rows, cols) if dx == "dx" else dx
    return lambda: b.donerf_train_distill(None, x if x else mat(F32, rows, cols), classes if classes else ints(I32, rows, k),
                                          teacher if teacher else mat(F32, rows, k), weight, temperature, loss, dx, rows, cols, k)


@pytest.mark.parametrize("call", [
    norm(), norm(weight=None, bias=None), norm(y=None), norm(kept=None), norm(x=mat(BF16, 4, 100, data=A + 2, ld=101)), norm(rows=0, stats=None),
    norm(rows=(1 << 31) - 1), norm(cols=1), norm(cols=b.MAX_COLS), norm(eps=1e-30),
    norm_backward(), norm_backward(dx=None), norm_backward(dw=None), norm_backward(db=None, dw=None), norm_backward(weight=None, x=mat(F32, 4, 100)),
    norm_backward(rows=0, stats=None), lookup(), lookup(ids=ints(I32, 4, 1, ld=9)), lookup(n=(1 << 31) - 1), lookup(rows=0),
    lookup_backward(), lookup_backward(rows=0, ws=None, ws_bytes=0), lookup_backward(accumulate=1, ids=ints(I64, 4, 1)),
    distill(), distill(weight=None, loss=None), distill(dx=None), distill(k=b.MAX_TOP), distill(cols=2, k=5), distill(rows=0),
    distill(temperature=2.0 ** -16), distill(temperature=2.0 ** 16), distill(classes=ints(I64, 4, 3, ld=8), teacher=mat(BF16, 4, 3, ld=5))])
def test_good_arguments_get_as_far_as_the_handle(call):
    refused(call, "handle is NULL")


MATRICES = [
    (lambda m: norm(x=m), "x", F32, 4, 100), (lambda m: norm(y=m), "y", BF16, 4, 100), (lambda m: norm(kept=m), "kept", b.MXFP8, 4, 100),
    (lambda m: norm_backward(dz=m), "dz", F32, 4, 100), (lambda m: norm_backward(x=m), "x", b.MXFP8, 4, 100),
    (lambda m: norm_backward(dx=m), "dx", BF16, 4, 100), (lambda m: lookup(table=m), "table", F32, 7, 100),
    (lambda m: lookup(ids=m), "ids", I32, 4, 1), (lambda m: lookup(ids=m), "ids", I64, 4, 1), (lambda m: lookup(y=m), "y", BF16, 4, 100),
    (lambda m: lookup_backward(dy=m), "dy", F32, 4, 100), (lambda m: lookup_backward(dtable=m), "dtable", F32, 7, 100),
    (lambda m: distill(x=m), "x", BF16, 4, 100), (lambda m: distill(classes=m), "classes", I64, 4, 3),
    (lambda m: distill(teacher=m), "teacher", F32, 4, 3), (lambda m: distill(dx=m), "dx", F32, 4, 100),
]


@pytest.mark.parametrize("call,name,kind,rows,cols", MATRICES)
def test_bad_matrices(call, name, kind, rows, cols):
    make = ints if kind in (I32, I64) else mat
    good = make(kind, rows, cols)
    refused(call(good), "handle is NULL")
    step = {F32: 4, BF16: 2, I32: 4, I64: 8}.get(kind, 16)
    bad = [({"data": None}, "NULL buffer"), ({"data": A + step // 2}, "not aligned"), ({"ld": good[1] - 1}, "ld out of range"),
           ({"ld": 0}, "ld out of range"), ({"ld": 1 << 41}, "ld out of range"), ({"type": 6}, "type is not taken"), ({"type": -1}, "type is not taken")]
    bad += [({"scales": A}, "scales given")] if kind != b.MXFP8 else [({"scales": None}, "NULL buffer")]
    for kw, message in bad:
        refused(call(make(kind, rows, cols, **kw)), f"{name}: ")
        refused(call(make(kind, rows, cols, **kw)), message)


@pytest.mark.parametrize("call,kinds", [
    (lambda m: norm(x=m), (b.MXFP4, b.MXFP8, I32)), (lambda m: norm(y=m), (b.MXFP8, I64)), (lambda m: norm(kept=m), (F32, b.MXFP4)),
    (lambda m: norm_backward(dz=m), (b.MXFP8, I32)), (lambda m: norm_backward(x=m), (b.MXFP4, I32)), (lambda m: norm_backward(dx=m), (b.MXFP8,)),
    (lambda m: lookup(table=m), (b.MXFP4, b.MXFP8, I32)), (lambda m: lookup(ids=m), (F32, BF16)), (lambda m: lookup(y=m), (b.MXFP8, I32)),
    (lambda m: lookup_backward(dy=m), (b.MXFP8, I32)), (lambda m: lookup_backward(dtable=m), (BF16, I32)),
    (lambda m: distill(x=m), (b.MXFP8, I32)), (lambda m: distill(classes=m), (F32, BF16)), (lambda m: distill(teacher=m), (I32, b.MXFP4)),
    (lambda m: distill(dx=m), (b.MXFP8, I64))])
def test_types_that_are_not_taken(call, kinds):
    for kind in kinds:
        m = ints(kind, 100, 100) if kind in (I32, I64) else mat(kind, 100, 100)
        refused(call(m), "type is not taken")


@pytest.mark.parametrize("make", [norm, norm_backward, lookup, lookup_backward, distill])
def test_sizes(make):
    for rows, cols in ((-1, 8), (1 << 31, 8), (4, 0), (4, -3), (4, b.MAX_COLS + 1)):
        refused(make(rows=rows, cols=cols), "must lie in")


def test_values():
    for eps in (0.0, -1.0, 1e-31, math.inf, math.nan):
        refused(norm(eps=eps), "eps must be")
    for t in (0.0, -1.0, 2.0 ** -17, 2.0 ** 17, math.inf, math.nan):
        refused(distill(temperature=t), "temperature must lie")
    for make in (lookup, lookup_backward):
        for n in (0, -1, 1 << 31):
            refused(make(n=n), "table rows must lie")
    for k in (0, -1, b.MAX_TOP + 1):
        refused(distill(k=k), "entries must lie")


def test_vectors_flags_and_what_is_missing():
    for make in (norm, norm_backward):
        refused(make(weight=A + 2), "weight not aligned")
        refused(make(stats=A + 4), "stats not aligned")
        refused(make(stats=None), "stats is NULL")
        refused(make(relu=2), "relu")
    refused(norm(bias=A + 1), "bias not aligned")
    refused(norm(y=None, kept=None), "neither y nor kept")
    refused(norm_backward(dw=A + 2), "dw not aligned")
    refused(norm_backward(db=A + 2), "db not aligned")
    refused(norm_backward(accumulate=-1), "must be 0 or 1")
    refused(norm_backward(dx=None, dw=None, db=None), "no gradient")
    refused(lookup_backward(accumulate=2), "must be 0 or 1")
    refused(distill(weight=A + 2), "row_weight not aligned")
    refused(distill(loss=A + 2), "loss not aligned")
    refused(distill(loss=None, dx=None), "neither loss nor dx")
    refused(lookup_backward(rows=1025, ws=None), "workspace is NULL")
    refused(lookup_backward(rows=1025, ws=A + 8), "workspace not aligned")
    refused(lookup_backward(rows=1025, ws_bytes=8), "workspace of", b.E_SIZE)
    refused(lookup_backward(rows=1024, ws=None, ws_bytes=0), "handle is NULL")      # needs none


def test_offsets_that_64_bits_would_not_hold():
    rows = (1 << 31) - 1
    refused(norm(rows=rows, cols=8, x=mat(F32, rows, 8, ld=1 << 40)), "x: ld out of range")
    refused(lookup(n=rows, cols=8, table=mat(F32, rows, 8, ld=1 << 40)), "table: ld out of range")


def test_workspaces_without_a_handle():
    assert b.donerf_train_norm_backward_workspace(None, 4, 4) == 0 == b.donerf_train_embedding_backward_workspace(None, 4, 4, 4)


def test_matrix_arguments_are_the_structure():
    for m in ((A, 100, b.TYPE_BF16), (A, 1 << 40, b.MXFP8, A + 64, 8), (None, 1, b.TYPE_INT64)):
        data, ld, kind, scales, ld_scales = m if len(m) == 5 else (*m, None, 0)
        assert b._mat(m) == bytes(b.donerf_mat(data, ld, scales, ld_scales, kind))
    assert b._mat(None) is None


def test_every_finite_eps_is_taken():
    for eps in (1e-30, 1.0, 3e38, 3.1e38, 3.4028234663852886e38):
        refused(norm(eps=eps), "handle is NULL")
