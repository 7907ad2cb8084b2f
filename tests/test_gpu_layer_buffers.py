"""What the layer operators write shares memory with nothing else of their call: the
scales of outputs and inputs, vectors and the workspace count like the matrices'
data, and buffers that only touch are taken.  Through the C names."""
import pytest
import torch

from paper_2103_03231_amd import binding as b
from paper_2103_03231_amd import inputs

pytestmark = pytest.mark.gpu
ROWS, IN, OUT = 70, 96, 64           # more rows than a product without a workspace takes
BF, F32 = b.TYPE_BF16, b.TYPE_FP32


@pytest.fixture(scope="module")
def r():
    r = b.Renderer(b.Config(), inputs.make_weights(128, 0))
    yield r
    r.close()


class Arena:
    """Addresses in one buffer, 64 KiB apart, so that any two may be put on each other."""

    def __init__(self):
        self.bytes = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")

    def at(self, slot, off=0):
        return self.bytes.data_ptr() + (slot << 16) + off


def mx(data, scales, cols, kind, ld=None, ld_scales=8):
    return data, ld or -(-cols // 32) * (16 if kind == b.MXFP4 else 32), kind, scales, ld_scales


def linear(r, a, **kw):
    p = {"x": a.at(0), "xs": a.at(1), "w": a.at(2), "ws": a.at(3), "y": a.at(4), "ys": a.at(5), "bias": a.at(6), "work": a.at(7), "kind": b.MXFP4}
    p.update(kw)
    x = mx(p["x"], p["xs"], IN, b.MXFP4) if p["kind"] == b.MXFP4 else (p["x"], IN, p["kind"])
    need = b.donerf_mx_linear_workspace(p["kind"], ROWS, IN)
    b.donerf_mx_linear(r.h, x, mx(p["w"], p["ws"], IN, b.MXFP4), p["bias"], 0, mx(p["y"], p["ys"], OUT, b.MXFP4), ROWS, IN, OUT,
                       p["work"] if need else None, need)


def forward(r, a, **kw):
    p = {"x": a.at(0), "w": a.at(1), "y": a.at(2), "k": a.at(3), "ks": a.at(4), "bias": a.at(5)}
    p.update(kw)
    b.donerf_train_linear(r.h, (p["x"], IN, BF), (p["w"], IN, BF), p["bias"], 0, (p["y"], OUT, BF), mx(p["k"], p["ks"], OUT, b.MXFP8), ROWS, IN, OUT)


def backward(r, a, rows=ROWS, **kw):
    p = {"dz": a.at(0), "x": a.at(2), "xs": a.at(4), "w": a.at(5), "dx": a.at(6), "dw": a.at(9), "db": a.at(10), "work": a.at(11)}
    p.update(kw)
    need = b.donerf_train_linear_backward_workspace(r.h, rows, IN, OUT)
    assert need <= 5 << 16       # the slots from the workspace's on
    b.donerf_train_linear_backward(r.h, (p["dz"], OUT, BF), mx(p["x"], p["xs"], IN, b.MXFP8), 1, (p["w"], IN, BF), (p["dx"], IN, BF),
                                   (p["dw"], IN, F32), p["db"], 0, rows, IN, OUT, p["work"], need)


LINEAR = [dict(ys=0), dict(ys=1), dict(ys=2), dict(ys=3), dict(ys=4), dict(ys=6), dict(y=1), dict(y=3), dict(y=6),
          dict(kind=BF, work=0), dict(kind=BF, work=2), dict(kind=BF, work=3), dict(kind=BF, work=4), dict(kind=BF, work=5), dict(kind=F32, work=6)]
FORWARD = [dict(ks=0), dict(ks=1), dict(ks=2), dict(ks=3), dict(ks=5), dict(k=5), dict(y=5), dict(y=4)]
BACKWARD = [dict(db=0), dict(db=2), dict(db=4), dict(db=5), dict(db=6), dict(db=9), dict(dx=4), dict(dw=4), dict(dw=10),
            *(dict(work=s, rows=200) for s in (0, 2, 4, 5, 6, 9, 10))]


@pytest.mark.parametrize("call,bad", [*((linear, k) for k in LINEAR), *((forward, k) for k in FORWARD), *((backward, k) for k in BACKWARD)],
                         ids=lambda v: v.__name__ if callable(v) else "-".join(f"{k}{n}" for k, n in v.items()))
def test_what_is_written_shares_nothing(r, call, bad):
    a = Arena()
    # 16 bytes further: within the other's first row
    moved = {k: v if k in ("kind", "rows") else a.at(v, 16) for k, v in bad.items()}
    with pytest.raises(b.DonerfError, match="overlaps another matrix or buffer") as e:
        call(r, a, **moved)
    assert e.value.status == b.E_INVALID_ARG
    torch.cuda.synchronize()
    assert (a.bytes == 0).all()
    apart = {k: v for k, v in bad.items() if k in ("kind", "rows")}
    call(r, a, **apart)
    torch.cuda.synchronize()


def test_conversions(r):
    a = Arena()
    for at in (a.at(0, 16), a.at(1, 16)):           # scales on x, on the codes
        with pytest.raises(b.DonerfError, match="q overlaps"):
            b.donerf_mx_quantize(r.h, (a.at(0), IN, BF), mx(a.at(1), at, IN, b.MXFP8), ROWS, IN)
    with pytest.raises(b.DonerfError, match="y overlaps"):
        b.donerf_mx_dequantize(r.h, mx(a.at(0), a.at(1, 64), IN, b.MXFP8), (a.at(1), IN, F32), ROWS, IN)


def test_neighbours_are_taken(r):
    """One buffer after the other, and records of codes and scales side by side."""
    x, w, bias = torch.randn(ROWS, IN, device="cuda").bfloat16(), torch.randn(OUT, IN, device="cuda").bfloat16(), torch.randn(OUT, device="cuda")
    y, kept = r.train_linear(x, w, bias)
    record = torch.full((ROWS, 80), 7, dtype=torch.uint8, device="cuda")       # 64 codes, 8 bytes of scales, 8 of the user's
    at = record.data_ptr()
    b.donerf_train_linear(r.h, (x.data_ptr(), IN, BF), (w.data_ptr(), IN, BF), bias.data_ptr(), 0, None,
                          mx(at, at + 64, OUT, b.MXFP8, 80, 80), ROWS, IN, OUT)
    assert torch.equal(record[:, :64], kept.codes) and torch.equal(record[:, 64:66], kept.scales[:, :2]) and (record[:, 66:] == 7).all()
    # scales in the place of the last codes
    with pytest.raises(b.DonerfError, match="kept overlaps"):
        b.donerf_train_linear(r.h, (x.data_ptr(), IN, BF), (w.data_ptr(), IN, BF), bias.data_ptr(), 0, None,
                              mx(at, at + 56, OUT, b.MXFP8, 80, 80), ROWS, IN, OUT)
    dz = torch.randn(200, OUT, device="cuda").bfloat16()
    x = torch.randn(200, IN, device="cuda").bfloat16()
    ref = r.train_linear_backward(dz, x, w)
    need = b.donerf_train_linear_backward_workspace(r.h, 200, IN, OUT)
    assert need > 0 and need % 4 == 0
    flat = torch.full((OUT * IN + OUT + need // 4 + 1,), 7.0, device="cuda")   # dw, db and the workspace without a gap
    at = flat.data_ptr()
    b.donerf_train_linear_backward(r.h, (dz.data_ptr(), OUT, BF), (x.data_ptr(), IN, BF), 0, None, None, (at, IN, F32), at + 4 * OUT * IN, 0,
                                   200, IN, OUT, at + 4 * (OUT * IN + OUT), need)
    assert torch.equal(flat[:OUT * IN].view(OUT, IN), ref[1]) and torch.equal(flat[OUT * IN:OUT * IN + OUT], ref[2]) and flat[-1] == 7


def test_sizes_that_are_refused_need_no_workspace(r):
    """What donerf_train_linear_backward refuses for its size, though its columns and
    rows alone lie in their ranges."""
    most = b.MAX_COLS
    for rows, n_in, n_out in (((1 << 31) - 1, most, most), ((1 << 31) - 1, most, 1), ((1 << 31) - 1, 1, most), (1 << 22, most, 8), (1 << 22, 8, most),
                              (-1, 8, 8), (8, 0, 8), (8, 8, most + 1)):
        assert b.donerf_train_linear_backward_workspace(r.h, rows, n_in, n_out) == 0, (rows, n_in, n_out)
    # taken: more tiles than the chip holds workgroups make one part, a single tile many
    need = lambda *size: b.donerf_train_linear_backward_workspace(r.h, *size)
    assert need((1 << 22) - 128, 8, most) == 0 < need(1 << 21, 8, 8) and need(1 << 21, 8, 8) % (4 * (8 * 8 + 8)) == 0
