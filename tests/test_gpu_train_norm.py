"""Layer norm forward and backward against the oracle and against differences,
through the public entry points.

A row's sum goes through at most 64 values of a lane, 7 of single columns, 6
exchanges and 16 waves: below 100 roundings of u = 2^-24 of the terms' summed
magnitudes.  Its other operations round once each, and the reciprocal square root is
off by at most a step, 2u.  bf16 results are off by half a bf16 step more, and what
is kept by half an E4M3 step at its block's scale."""
import numpy as np
import pytest
import torch

from oracle import layers_oracle as L
from oracle import training_oracle as O
from paper_2103_03231_amd import binding as b
from paper_2103_03231_amd import inputs
from test_gpu_mx import device, host, numbers

pytestmark = pytest.mark.gpu
U, SUM = 2.0 ** -24, 100 * 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2}
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def r():
    r = b.Renderer(b.Config(), inputs.make_weights(128, 0))
    yield r
    r.close()


def f64(t):
    return t.double().cpu().numpy()


def normal(seed, *shape, scale=1.0, dtype=F32, pad=0):
    """A tensor whose rows are `pad` values further apart than they are long."""
    g = torch.Generator().manual_seed(seed)
    wide = (*shape[:-1], shape[-1] + pad)
    return (torch.randn(*wide, generator=g) * scale).to(dtype).cuda()[..., :shape[-1]]


def rows_of(seed, rows, cols, dtype=F32, pad=0, relu=False):
    """Rows of different sizes around a mean of their own."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, cols + pad, generator=g) + 0.5 * torch.randn(rows, 1, generator=g)) * torch.exp(torch.randn(rows, 1, generator=g))
    return (torch.relu(x) if relu else x).to(dtype).cuda()[:, :cols]


def forward_bounds(x, w, bias, eps):
    """(of z, of the mean, of r)."""
    n = x.shape[1]
    mean, r = O.norm_stats(x, eps).T[:, :, None]
    d = np.abs(x - mean)
    em = (SUM + 4 * U) * np.abs(x).sum(1, keepdims=True) / n
    var = (d ** 2).mean(1, keepdims=True)
    ev = 2 * em * d.mean(1, keepdims=True) + em ** 2 + (SUM + 8 * U) * (var + 2 * em * d.mean(1, keepdims=True) + em ** 2) + 2 * U * eps
    rel = ev * r ** 2
    assert (rel < 0.1).all(), "inputs for which the bound says nothing"
    er = r * (0.5 * rel / (1 - rel) ** 1.5 + 3 * U)
    z = ((d + em) * (r + er) - d * r) + 3 * U * (d + em) * (r + er)
    if w is not None:
        z = z * np.abs(w)
    full = (d + em) * (r + er) * (1.0 if w is None else np.abs(w)) + (0.0 if bias is None else np.abs(bias))
    return z + 3 * U * full, em, er


def check_forward(r, x, w, bias, relu, out=BF16, eps=1e-5):
    vx, vw, vb = f64(x), None if w is None else f64(w), None if bias is None else f64(bias)
    ref = O.norm(vx, vw, vb, eps, relu)
    tol, em, er = forward_bounds(vx, vw, vb, eps)
    y, kept, stats = r.train_norm(x, w, bias, eps=eps, relu=relu, out=out)
    assert y.dtype is out
    got = f64(y)
    assert (np.abs(got - ref) <= tol + HALF[out] * (np.abs(ref) + tol)).all(), np.abs(got - ref).max()
    st = f64(stats)
    mean, rr = O.norm_stats(vx, eps).T[:, :, None]
    assert (np.abs(st[:, :1] - mean) <= em + U * np.abs(mean)).all() and (np.abs(st[:, 1:] - rr) <= er).all()
    _, scales = host(kept)
    v = numbers(kept)
    assert (np.abs(v - ref) <= L.half_step(np.abs(ref) + tol, scales, "mxfp8") + tol).all()
    # whole blocks, zeros behind the last column, and no larger a scale than needed
    codes = kept.codes.cpu().numpy()
    assert (codes[:, x.shape[1]:] == 0).all()
    blocks = -(-ref.shape[1] // 32)
    pad = lambda a: np.pad(np.broadcast_to(a, ref.shape), ((0, 0), (0, blocks * 32 - ref.shape[1]))).reshape(len(ref), blocks, 32).max(2)
    top, slack = pad(np.abs(ref)), pad(tol)
    full = 448 * np.exp2(scales.astype(float) - 127)
    assert (top <= full + slack).all() and ((top + slack >= full / 2 * (1 - 1e-6)) | (scales == 0)).all()
    if out is F32 and not relu:      # the checkpoint is made of the same fp32 values
        q = r.mx_quantize(y, b.MXFP8)
        assert torch.equal(q.codes, kept.codes) and torch.equal(q.scales[:, :blocks], kept.scales[:, :blocks])
    y2, none, stats2 = r.train_norm(x, w, bias, eps=eps, relu=relu, keep=False, out=out)
    assert none is None and torch.equal(y, y2) and torch.equal(stats, stats2)


SIZES = [(1, 1), (3, 2), (5, 7), (1, 8), (2, 9), (13, 31), (40, 32), (33, 33), (70, 63), (65, 64), (9, 65), (200, 100), (31, 128), (30, 129),
         (300, 256), (1000, 255), (129, 257), (64, 283), (20, 512), (19, 513), (40, 1000), (16, 1024), (7, 1025), (12, 2048), (5, 2051),
         (6, 4096), (3, 4099), (4, 8192), (3, 8190), (2, 16384), (3, 16391), (2, 32768), (1, 32769), (2, 65536), (1, 65531)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(r, rows, cols, dtype):
    w, bias = 1 + normal(cols, cols, scale=0.2), normal(cols + 1, cols, scale=0.1)
    check_forward(r, rows_of(rows, rows, cols, dtype), w, bias, True)
    check_forward(r, rows_of(rows + 1, rows, cols, dtype, pad=5), w, None, False, out=F32)
    check_forward(r, rows_of(rows + 2, rows, cols, dtype, pad=3), None, bias, False)
    check_forward(r, rows_of(rows + 3, rows, cols, dtype), None, None, True, out=F32, eps=0.5)


def check_backward(r, dz, x, stats, w, relu, out=BF16):
    vx = numbers(x) if isinstance(x, b.MxTensor) else f64(x)
    zero = None
    if relu:
        zero = host(x)[0].reshape(vx.shape[0], -1)[:, :vx.shape[1]] % 128 == 0 if isinstance(x, b.MxTensor) else vx == 0
    vz, st, vw = f64(dz), f64(stats), None if w is None else f64(w)
    rx, rw, rb = O.norm_backward(vz, vx, st, vw, zero)
    dx, dw, db = r.train_norm_backward(dz, x, stats, w, relu=relu, out=out)
    assert dx.dtype is out
    rows, n = vz.shape
    xh = np.abs((vx - st[:, :1]) * st[:, 1:])
    g = np.abs(vz if vw is None else vz * vw)
    c1, c2 = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    # sums of |terms| bound the means and their errors; xh is off by 2u, g by u, the means by 3u more each
    tol = st[:, 1:] * (4 * U * g + (SUM + 8 * U) * c1 + xh * (SUM + 12 * U) * c2 + 4 * U * (c1 + xh * c2))
    if relu:
        tol = np.where(zero, 0.0, tol)
    assert (np.abs(f64(dx) - rx) <= tol + HALF[out] * (np.abs(rx) + tol)).all(), np.abs(f64(dx) - rx).max()
    for got, ref, mag in ((dw, rw, (np.abs(vz) * xh).sum(0)), (db, rb, np.abs(vz).sum(0))):
        assert (np.abs(f64(got) - ref) <= (rows + 4) * U * mag).all()
    # the same bits, with and without the others
    again = r.train_norm_backward(dz, x, stats, w, relu=relu, out=out)
    assert all(torch.equal(u, v) for u, v in zip((dx, dw, db), again))
    none, dw2, db2 = r.train_norm_backward(dz, x, stats, w, relu=relu, need_dx=False)
    assert none is None and torch.equal(dw, dw2) and torch.equal(db, db2)
    acc = r.train_norm_backward(dz, x, stats, w, relu=relu, need_dx=False, dw=torch.full_like(dw, 0.5), db=torch.full_like(db, -2.0))
    assert torch.equal(acc[1], 0.5 + dw) and torch.equal(acc[2], -2.0 + db)


@pytest.mark.parametrize("kind", [F32, BF16, b.MXFP8], ids=str)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(r, rows, cols, kind):
    w = 1 + normal(cols, cols, scale=0.2)
    for seed, (dz_type, relu, pad, out, weight) in enumerate([(BF16, True, 0, BF16, w), (F32, False, 3, F32, None), (BF16, False, 5, F32, w)]):
        x = rows_of(rows + seed, rows, cols, BF16 if kind is BF16 else F32, 0 if kind == b.MXFP8 else pad, relu)
        stats = torch.from_numpy(O.norm_stats(f64(x), 1e-5)).float().cuda()
        if kind == b.MXFP8:
            x = r.mx_quantize(x, b.MXFP8)
        check_backward(r, normal(seed + 7, rows, cols, scale=1 / rows, dtype=dz_type, pad=pad), x, stats, weight, relu, out)


@pytest.mark.parametrize("rows,cols", [(20000, 64), (70001, 33), (5000, 1000), (3001, 2049), (4000, 130), (1025, 5000), (700, 12000), (600, 20001)])
def test_many_rows(r, rows, cols):
    """More rows than workgroups, in 64 bits on the GPU."""
    x = rows_of(1, rows, cols, BF16, relu=True)
    dz = normal(2, rows, cols, scale=1 / rows, dtype=BF16)
    w = 1 + normal(3, cols, scale=0.2)
    y, _, stats = r.train_norm(x, w, keep=False, out=F32)
    v = x.double()
    mean = v.mean(1, keepdim=True)
    rr = torch.rsqrt((v - mean).square().mean(1, keepdim=True) + 1e-5)
    # z's error by the bounds above, with |x| <= |d| + |mean|: SUM (mean|x|) r each in the mean, and in r by half of twice that
    tol = (2 * SUM + 16 * U) * (1 + ((v - mean) * rr).abs()) * (1 + v.abs().mean(1, keepdim=True) * rr) * w.abs()
    assert ((y.double() - (v - mean) * rr * w).abs() <= tol).all()
    for x_in in (x, r.mx_quantize(x, b.MXFP8)):
        v = x.double() if x_in is x else r.mx_dequantize(x_in, F32).double()
        dx, dw, db = r.train_norm_backward(dz, x_in, stats, w, relu=True, out=F32)
        xh, z = (v - stats[:, :1].double()) * stats[:, 1:].double(), dz.double()
        g = z * w.double()
        ref = stats[:, 1:].double() * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * (v != 0)
        tol = stats[:, 1:].double() * (8 * U * g.abs() + (SUM + 12 * U) * (g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True)))
        assert ((dx.double() - ref).abs() <= tol).all()
        # a column's sum: a row's share of the workgroups' rows, then their parts; the bound by rows holds
        for got, ref, mag in ((dw, (z * xh).sum(0), (z * xh).abs().sum(0)), (db, z.sum(0), z.abs().sum(0))):
            assert ((got.double() - ref).abs() <= (rows + 4) * U * mag).all()
            # and in the norm, where roundings of either sign average out: 16 in a row of half a step, each at full size
            assert torch.linalg.norm(got.double() - ref) <= 16 * U * torch.linalg.norm(mag)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(66001, 61), (66001, 100), (33001, 250), (16500, 507), (8300, 1001), (4200, 2043), (2100, 4090), (1100, 8191),
                                       (1100, 12003), (600, 20007), (600, 33001)])
def test_rows_of_a_workgroup_after_its_first(r, rows, cols, dtype):
    """Rows are independent of each other: a call that gives each workgroup several has the bits of calls that give it one."""
    x, w, bias = rows_of(1, rows, cols, dtype, pad=1), 1 + normal(2, cols, scale=0.2), normal(3, cols)
    y, kept, stats = r.train_norm(x, w, bias, relu=True)
    dz = normal(4, rows, cols, dtype=BF16)
    dx, _, _ = r.train_norm_backward(dz, x, stats, w)
    per = rows // 5 + 1
    for at in range(0, rows, per):
        part = slice(at, at + per)
        y2, kept2, stats2 = r.train_norm(x[part], w, bias, relu=True)
        assert torch.equal(y[part], y2) and torch.equal(stats[part], stats2)
        blocks = (cols + 31) // 32
        assert torch.equal(kept.codes[part, :cols], kept2.codes[:, :cols]) and torch.equal(kept.scales[part, :blocks], kept2.scales[:, :blocks])
        assert torch.equal(dx[part], r.train_norm_backward(dz[part], x[part], stats2, w)[0])


def test_gradient_against_differences(r):
    """The whole way, forwards and backwards, with fp32 rows: central differences of the forward pass in 64 bits."""
    x, w, bias, dz = rows_of(5, 4, 37), 1 + normal(6, 37, scale=0.2), normal(7, 37), normal(8, 4, 37)
    _, _, stats = r.train_norm(x, w, bias, keep=False)
    dx, dw, db = r.train_norm_backward(dz, x, stats, w, out=F32)
    vx, vw, vb, vz = (f64(t) for t in (x, w, bias, dz))

    def slope(f, v, step=1e-5):
        d = np.zeros(v.shape)
        for i in np.ndindex(v.shape):
            up, down = v.copy(), v.copy()
            up[i] += step
            down[i] -= step
            d[i] = (f(up) - f(down)) / (2 * step)
        return d

    # differences of step h are off by h^2 times the third derivative, and stats of fp32 by parts in 10^7
    for got, ref in ((dx, slope(lambda v: (O.norm(v, vw, vb) * vz).sum(), vx)), (dw, slope(lambda v: (O.norm(vx, v, vb) * vz).sum(), vw)),
                     (db, slope(lambda v: (O.norm(vx, vw, v) * vz).sum(), vb))):
        assert np.abs(f64(got) - ref).max() <= 1e-5 * np.abs(ref).max()


def test_rows_of_one_value_and_of_one_column(r):
    x = torch.full((3, 40), 1e30, device="cuda")
    x[1], x[2] = -3.0, 0.0
    bias = normal(1, 40)
    y, kept, stats = r.train_norm(x, None, bias, out=F32)
    # the mean of equal values is theirs: r = 1 / sqrt(eps), z = bias
    assert torch.equal(stats[:, 0], x[:, 0]) and torch.allclose(stats[:, 1], torch.full((3,), 1e-5 ** -0.5, device="cuda"), rtol=4 * U, atol=0)
    assert torch.equal(y, bias.expand(3, 40))
    dz = normal(2, 3, 40)
    dx, dw, db = r.train_norm_backward(dz, x, stats, None, out=F32)
    assert (dw == 0).all() and torch.isfinite(dx).all()
    y, _, stats = r.train_norm(normal(3, 5, 1), torch.full((1,), 2.0, device="cuda"), torch.full((1,), 0.25, device="cuda"), out=F32)
    assert (y == 0.25).all()


def test_what_is_not_finite_stays_in_its_row(r):
    x = rows_of(9, 12, 70)
    dz = normal(3, 12, 70)
    y, kept, stats = r.train_norm(x, out=F32)
    dx, _, _ = r.train_norm_backward(dz, x, stats, out=F32)
    bad = x.clone()
    bad[2, 5], bad[4, 69], bad[7, 64] = float("nan"), float("inf"), -float("inf")
    yb, kb, sb = r.train_norm(bad, relu=False, out=F32)
    rows = [2, 4, 7]
    good = [i for i in range(12) if i not in rows]
    assert torch.isnan(yb[rows]).all() and torch.equal(yb[good], y[good]) and torch.equal(kb.codes[good], kept.codes[good])
    assert torch.isnan(r.mx_dequantize(kb, F32)[rows]).all()
    dxb, dw, db = r.train_norm_backward(dz, bad, sb, out=F32)
    assert torch.isnan(dxb[rows]).all() and torch.equal(dxb[good], dx[good]) and torch.isfinite(db).all()
    assert torch.isnan(r.train_norm(bad, relu=True, out=F32)[0][rows]).all()       # kept by the ReLU


def test_zeros_of_blocks_whose_scale_is_nan_stop_the_gradient(r):
    x = r.mx_quantize(rows_of(2, 3, 64, relu=True), b.MXFP8)
    x.scales[1, 0] = 255
    zero = torch.from_numpy(host(x)[0].reshape(3, 64) % 128 == 0).cuda()
    dx, _, _ = r.train_norm_backward(normal(1, 3, 64), x, torch.ones(3, 2, device="cuda"), relu=True, out=F32)
    assert (dx[zero] == 0).all() and torch.isnan(dx[1][~zero[1]]).all() and torch.isfinite(dx[[0, 2]]).all()


def test_no_rows(r):
    x = torch.empty(0, 5, device="cuda")
    y, kept, stats = r.train_norm(x)
    assert y.shape == (0, 5) and kept.rows == 0 and stats.shape == (0, 2)
    dx, dw, db = r.train_norm_backward(x, x, stats)
    assert dx.shape == (0, 5) and (dw == 0).all() and (db == 0).all()
    dw, db = torch.full((5,), 3.0, device="cuda"), torch.full((5,), 4.0, device="cuda")
    r.train_norm_backward(x, x, stats, dw=dw, db=db)
    assert (dw == 3).all() and (db == 4).all()


def test_what_lies_between_the_rows_stays(r):
    """Outputs in wider buffers, through the C names, in every type."""
    rows, cols = 37, 45
    x, w = rows_of(1, rows, cols), normal(2, cols)
    y, kept, stats = r.train_norm(x, w, out=F32)
    dz = normal(3, rows, cols)
    dx, dw, db = r.train_norm_backward(dz, x, stats, w, out=F32)
    for dtype, kind in ((F32, b.TYPE_FP32), (BF16, b.TYPE_BF16)):
        wide = torch.full((rows, cols + 3), 7.0, dtype=dtype, device="cuda")
        codes, scales = torch.full((rows, 96), 9, dtype=torch.uint8, device="cuda"), torch.full((rows, 16), 9, dtype=torch.uint8, device="cuda")
        st = torch.empty(rows, 2, device="cuda")
        b.donerf_train_norm(r.h, (x.data_ptr(), cols, b.TYPE_FP32), w.data_ptr(), None, 1e-5, 0, (wide.data_ptr(), cols + 3, kind),
                            (codes.data_ptr(), 96, b.MXFP8, scales.data_ptr(), 16), st.data_ptr(), rows, cols)
        assert torch.equal(wide[:, :cols], y.to(dtype)) and (wide[:, cols:] == 7).all() and torch.equal(st, stats)
        assert torch.equal(codes[:, :64], kept.codes) and (codes[:, 64:] == 9).all()
        assert torch.equal(scales[:, :2], kept.scales[:, :2]) and (scales[:, 2:] == 9).all()
        wide.fill_(7.0)
        b.donerf_train_norm_backward(r.h, (dz.data_ptr(), cols, b.TYPE_FP32), (x.data_ptr(), cols, b.TYPE_FP32), 0, w.data_ptr(), stats.data_ptr(),
                                     (wide.data_ptr(), cols + 3, kind), None, None, 0, rows, cols)
        assert torch.equal(wide[:, :cols], dx.to(dtype)) and (wide[:, cols:] == 7).all()


def test_refusals(r):
    x, v = rows_of(1, 8, 32), normal(1, 32)
    y, kept, stats = r.train_norm(x, v)
    for call in (lambda: r.train_norm(x.half()), lambda: r.train_norm(x.cpu()), lambda: r.train_norm(x.t()), lambda: r.train_norm(x[0]),
                 lambda: r.train_norm(x, v[:31]), lambda: r.train_norm(x, v.double()), lambda: r.train_norm(x, v, v.cpu()),
                 lambda: r.train_norm(x, out=torch.float16), lambda: r.train_norm_backward(x, x, stats[:7]), lambda: r.train_norm_backward(x, x, stats.t()),
                 lambda: r.train_norm_backward(x, x[:, :31], stats), lambda: r.train_norm_backward(x, r.mx_quantize(x, b.MXFP4), stats),
                 lambda: r.train_norm_backward(x, kept, stats, dw=v), lambda: r.train_norm_backward(x, kept, stats, dw=v[:31], db=v)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(b.DonerfError, match="eps"):
        r.train_norm(x, eps=0.0)
    for shares in (dict(dw=v, db=v), ):
        with pytest.raises(b.DonerfError, match="overlaps"):
            r.train_norm_backward(x, x, stats, **shares)
    with pytest.raises(b.DonerfError, match="stats overlaps"):
        b.donerf_train_norm(r.h, (x.data_ptr(), 32, b.TYPE_FP32), None, None, 1e-5, 0, (y.data_ptr(), 32, b.TYPE_BF16), None, x.data_ptr(), 8, 32)
    with pytest.raises(b.DonerfError, match="dx overlaps"):
        b.donerf_train_norm_backward(r.h, (x.data_ptr(), 32, b.TYPE_FP32), (y.data_ptr(), 32, b.TYPE_BF16), 0, None, stats.data_ptr(),
                                     (x.data_ptr(), 32, b.TYPE_FP32), None, None, 0, 8, 32)
    v = torch.zeros(3000 * 32, device="cuda")
    need = b.donerf_train_norm_backward_workspace(r.h, 3000, 32)
    assert need > 0 == b.donerf_train_norm_backward_workspace(r.h, 2048, 32)
    for ws, size, what in ((None, need, "workspace is NULL"), (v.data_ptr() + 8, need, "workspace not aligned"), (v.data_ptr(), need - 1, "workspace of")):
        with pytest.raises(b.DonerfError, match=what):
            b.donerf_train_norm_backward(r.h, (v.data_ptr(), 32, b.TYPE_FP32), (v.data_ptr(), 32, b.TYPE_FP32), 0, None, v.data_ptr(), None, y.data_ptr(), None,
                                         0, 3000, 32, ws, size)
    with torch.cuda.stream(torch.cuda.Stream()):
        with pytest.raises(ValueError, match="stream"):
            r.train_norm(x)


BIG = torch.finfo(F32).max


@pytest.mark.parametrize("cols", [1, 3, 8, 40, 61, 283, 1000, 2051, 4096, 9001, 16385, 32000, 65536])
def test_rows_whose_sums_and_squares_do_not_fit(r, cols):
    """Finite rows of any size: of one value they are exact; of values whose squares overflow r is 0, and z the bias."""
    half = cols - cols // 2
    x = rows_of(1, 10, cols)
    plain, kept0, stats0 = r.train_norm(x[7:], None, None, out=F32)
    x[0], x[1], x[2] = 1e38, -BIG, BIG
    x[3] = normal(2, cols) * 1e37                                          # squares
    x[4] = 3e38
    x[4, half:] = -3e38                                                    # differences, too
    x[5] = -1e30
    x[5, 0] = 2e30
    x[6] = 3e38                                                            # and the sum
    x[6, 0] = 2.5e38
    bias = normal(3, cols)
    mean = x.double().mean(1)
    overflow = (x.double() - mean[:, None]).square().sum(1) > float(BIG)
    for dtype in (F32, BF16):
        v = x.to(dtype)
        if dtype is BF16:
            v[1], v[2] = torch.finfo(BF16).min, torch.finfo(BF16).max
        mean = v.double().mean(1)
        y, kept, stats = r.train_norm(v, None, bias, out=F32)
        one = [0, 1, 2] if cols > 1 else list(range(7))
        assert torch.equal(stats[one, 0], v[one, 0].float()) and torch.allclose(stats[one, 1], torch.full((len(one),), 1e-5 ** -0.5, device="cuda"), rtol=4 * U, atol=0)
        assert torch.equal(y[:7], bias.expand(7, cols)) or cols == 1
        assert torch.equal(y[one], bias.expand(len(one), cols))
        if cols > 1:
            assert (stats[3:7, 1] == 0).all() and overflow[3:7].all()
            # the mean, by the bound of a sum and its correction, with |x| summed; 0 where differences to it may overflow
            near = torch.where(mean[3:7].abs() < 2.0 ** 102, mean[3:7], 0)
            assert ((stats[3:7, 0].double() - near).abs() <= (2 * SUM + 8 * U) * v[3:7].double().abs().mean(1)).all()
        assert torch.isfinite(r.mx_dequantize(kept, F32)).all()
        if dtype is F32:
            again = r.train_norm(x[7:], None, None, out=F32)
            assert torch.equal(again[0], plain) and torch.equal(again[2], stats0) and torch.equal(stats[7:], stats0)
        # backwards: no part in dw, no gradient where r is 0
        dz = normal(4, 10, cols)
        for x_in in (v, r.mx_quantize(v.clamp(-1e38, 1e38), b.MXFP8)):
            dx, dw, db = r.train_norm_backward(dz, x_in, stats, None, out=F32)
            assert torch.isfinite(dx).all() or x_in is not v      # (8 bits do not hold the rows of one value)
            if cols > 1:
                assert (dx[3:7] == 0).all()
            if x_in is v:
                ref = r.train_norm_backward(dz[7:], v[7:], stats[7:], None, out=F32)
                assert torch.equal(dx[7:], ref[0]) and torch.isfinite(dw).all() and torch.isfinite(db).all()
                rest = (dz[7:].double() * (v[7:].double() - stats[7:, :1].double()) * stats[7:, 1:].double())
                assert ((dw.double() - rest.sum(0)).abs() <= 14 * U * rest.abs().sum(0)).all()


def test_many_rows_whose_squares_do_not_fit(r):
    """In the kernels that add up dw on the way, and in those for columns."""
    for rows, cols in ((4000, 70), (3000, 2050), (2050, 20001)):
        x = rows_of(1, rows, cols, BF16)
        x[::3, ::2], x[::3, 1::2] = 3e38, -3e38
        x[::3, 0] = -3e38
        _, _, stats = r.train_norm(x, keep=False)
        dz = normal(2, rows, cols, dtype=BF16)
        dx, dw, db = r.train_norm_backward(dz, x, stats, out=F32)
        assert (stats[::3, 1] == 0).all() and torch.isfinite(stats).all() and (dx[::3] == 0).all() and torch.isfinite(dx).all()
        good = torch.ones(rows, dtype=torch.bool, device="cuda")
        good[::3] = False
        rest = dz[good].double() * (x[good].double() - stats[good, :1].double()) * stats[good, 1:].double()
        assert ((dw.double() - rest.sum(0)).abs() <= (rows + 4) * U * rest.abs().sum(0)).all()


def test_what_is_not_finite_is_not_taken_for_an_overflow(r):
    for cols in (3, 64, 283, 5000, 40000):
        x = rows_of(9, 5, cols)
        x[0, 1], x[1, cols - 1], x[2, 0] = float("inf"), -float("inf"), float("nan")
        x[3, 0], x[3, 1] = float("inf"), -float("inf")
        y, kept, stats = r.train_norm(x, out=F32)
        assert torch.isnan(y[:4]).all() and torch.isnan(stats[:4, 1]).all() and torch.isfinite(y[4]).all() and torch.isfinite(stats[4]).all()
        dx, dw, db = r.train_norm_backward(normal(3, 5, cols), x, stats, out=F32)
        assert torch.isnan(dx[:4]).all() and torch.isfinite(dx[4]).all() and torch.isnan(dw).all()


@pytest.mark.parametrize("rows,cols,one", [(2048, 2048, True), (2047, 2049, True), (2048, 2049, False), (2049, 2048, False), (1024, 4096, True),
                                           (1025, 4096, False), (2048, 4096, False), (2048, 4095, False), (2047, 4097, True), (2048, 4097, False),
                                           (1024, 8192, True), (1025, 8192, False), (512, 16384, True), (513, 16384, False), (419, 20000, True),
                                           (420, 20000, False), (128, 65536, True), (129, 65536, False), (2049, 8, False), (2048, 8, True)])
def test_gradients_on_either_side_of_one_launch(r, rows, cols, one):
    """dw and db by columns without a workspace, and as parts in one.  Whole numbers, whose sums are exact: both give the same."""
    assert (b.donerf_train_norm_backward_workspace(r.h, rows, cols) == 0) is one
    g = torch.Generator().manual_seed(rows)
    x = torch.randint(-8, 9, (rows, cols), generator=g, dtype=torch.int8).cuda()
    dz = torch.randint(-8, 9, (rows, cols), generator=g, dtype=torch.int8).cuda()
    stats = torch.stack([torch.randint(-3, 4, (rows,), generator=g).float(), torch.randint(1, 3, (rows,), generator=g).float()], 1).cuda()
    xh = (x.double() - stats[:, :1]) * stats[:, 1:]
    for dtype in (F32, BF16):
        _, dw, db = r.train_norm_backward(dz.to(BF16), x.to(dtype), stats, need_dx=False)
        assert torch.equal(dw.double(), (dz.double() * xh).sum(0)) and torch.equal(db.double(), dz.double().sum(0))
