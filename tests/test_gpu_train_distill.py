"""The distillation loss and its gradient against the oracle, through the public entry
points.

With A = |x - max| / T and B = |t - max| / T, an exponential is off by 3u (u = 2^-24) of
its argument from the difference, the scale and the product, and by a step, 2u, of its
own; a sum by below 100 roundings (64 values of a lane, 7 single ones, 6 exchanges, 16
waves).  Results below 2^-126 may become zero.  bf16 gradients are off by half a bf16
step more."""
import numpy as np
import pytest
import torch

from oracle import training_oracle as O
from paper_2103_03231_amd import binding as b
from paper_2103_03231_amd import inputs

pytestmark = pytest.mark.gpu
U, SUM, LEAST = 2.0 ** -24, 100 * 2.0 ** -24, 2.0 ** -126
HALF = {torch.float32: 0.0, torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2}
F32, BF16 = torch.float32, torch.bfloat16
INF = float("inf")


@pytest.fixture(scope="module")
def r():
    r = b.Renderer(b.Config(), inputs.make_weights(128, 0))
    yield r
    r.close()


def f64(t):
    return t.double().cpu().numpy()


def inputs_of(seed, rows, cols, k, dtype=F32, kind=torch.int64, pad=0, masked=False, twice=False):
    """(x, classes, teacher, row_weight): a teacher near the student; masked: classes of -inf, entries that are not given, rows
    without weight; twice: classes that come more than once."""
    g = torch.Generator().manual_seed(seed)
    x = 2 * torch.randn(rows, cols + pad, generator=g)
    near = x[:, :cols] + torch.randn(rows, cols, generator=g)
    if twice or k > cols:
        classes = torch.randint(0, max(1, cols // 2), (rows, k), generator=g)
        t = near.gather(1, classes) + torch.randn(rows, k, generator=g)
    else:
        t, classes = torch.topk(near, k, dim=1)
    weight = torch.rand(rows, generator=g) + 0.5
    if masked:
        off = (torch.rand(rows, cols, generator=g) < 0.3).scatter(1, classes, False)
        x[:, :cols][off] = -INF
        lost = torch.arange(k) >= (torch.rand(rows, 1, generator=g) * (k + 1)).floor()
        classes = torch.where(lost, torch.tensor([-1, cols, -5, 1 << 30])[torch.randint(0, 4, (rows, k), generator=g)], classes)
        t = torch.where(lost, torch.tensor([float("nan"), INF, -INF, 0.0])[torch.randint(0, 4, (rows, k), generator=g)], t)
        t = torch.where((torch.rand(rows, k, generator=g) < 0.1) & ~lost, -INF, t)
        weight = torch.where(torch.rand(rows, generator=g) < 0.2, 0.0, weight)
    return x.to(dtype).cuda()[:, :cols], classes.to(kind).cuda(), t.cuda(), weight.cuda()


def bounds(x, classes, t, temp, weight):
    """(of the loss, of dx) without a final rounding."""
    rows, cols = x.shape
    bl, bd = np.zeros(rows), np.zeros(x.shape)
    for i in range(rows):
        given = (classes[i] >= 0) & (classes[i] < cols)
        c, v = classes[i][given], t[i][given]
        if weight[i] == 0 or not (v > -np.inf).any() or not (x[i] > -np.inf).any():
            continue
        A, B = (x[i].max() - x[i]) / temp, (v.max() - v) / temp
        q, p = np.exp(-A), np.exp(-B)
        lq, lp = np.log(q.sum()), np.log(p.sum())
        q, p = q / q.sum(), p / p.sum()
        fa, fb = np.where(np.isfinite(A), A, 0.0), np.where(np.isfinite(B), B, 0.0)
        of_sum_q, of_sum_p = 4 * U * (q * fa).sum() + SUM + 3 * U, 4 * U * (p * fb).sum() + SUM + 3 * U
        rel_q, rel_p = 4 * U * fa + of_sum_q + 4 * U, 4 * U * fb + of_sum_p + 4 * U
        term = fa[c] + fb + lq + lp
        bl[i] = abs(weight[i]) * temp ** 2 * ((p * ((rel_p + SUM + 8 * U) * term + 4 * U * (fa[c] + fb))).sum() + of_sum_q + of_sum_p + 6 * U * (lq + lp))
        bd[i] = abs(weight[i]) * temp * ((rel_q + 4 * U) * q + LEAST)
        np.add.at(bd[i], c, abs(weight[i]) * temp * ((rel_p + (len(c) + 4) * U) * p + LEAST))
    return bl, bd


def check(r, x, classes, t, weight, temp, out=BF16):
    w = np.ones(len(x)) if weight is None else f64(weight)
    vx, vc, vt = f64(x), classes.cpu().numpy(), f64(t)
    ref_l, ref_d = O.distill(vx, vc, vt, temp, w)
    bl, bd = bounds(vx, vc, vt, temp, w)
    loss, dx = r.train_distill(x, classes, t, temperature=temp, row_weight=weight, out=out)
    assert dx.dtype is out and loss.dtype is F32
    assert (np.abs(f64(loss) - ref_l) <= bl + U * np.abs(ref_l)).all(), np.abs(f64(loss) - ref_l).max()
    assert (np.abs(f64(dx) - ref_d) <= bd + HALF[out] * (np.abs(ref_d) + bd)).all(), np.abs(f64(dx) - ref_d).max()
    assert (f64(loss)[bl == 0] == 0).all() and (f64(dx)[bl == 0] == 0).all()
    loss2, dx2 = r.train_distill(x, classes, t, temperature=temp, row_weight=weight, out=out)
    assert torch.equal(loss, loss2) and torch.equal(dx, dx2)              # the same bits
    loss3, none = r.train_distill(x, classes, t, temperature=temp, row_weight=weight, need_dx=False)
    assert none is None and torch.equal(loss, loss3)


SIZES = [(1, 1, 1), (2, 2, 2), (5, 7, 3), (1, 8, 8), (40, 9, 4), (33, 31, 1), (70, 64, 16), (300, 100, 4), (1000, 128, 4), (65, 129, 5), (257, 192, 7),
         (30, 256, 128), (300, 128, 128), (200, 64, 100), (100, 8, 64), (90, 24, 65), (20, 283, 33), (19, 512, 64), (9, 1000, 10), (7, 1024, 100), (5, 2048, 128), (4, 2055, 65), (3, 4096, 64), (2, 5001, 128),
         (3, 8192, 1), (2, 16384, 128), (2, 16390, 7), (2, 32000, 64), (1, 32768, 128), (2, 40001, 50), (1, 65536, 128), (1, 65535, 3)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,k", SIZES)
def test_loss_and_gradient(r, rows, cols, k, dtype):
    x, c, t, w = inputs_of(rows + cols, rows, cols, k, dtype)
    check(r, x, c, t, None, 1.0, F32)
    check(r, x, c, t.bfloat16(), w, 2.0)
    x, c, t, w = inputs_of(rows + cols + 1, rows, cols, k, dtype, torch.int32, pad=3, masked=True)
    check(r, x, c, t, w, 0.5, F32)
    x, c, t, w = inputs_of(rows + cols + 2, rows, cols, k, dtype, torch.int32, pad=1, twice=True)
    check(r, x, c, t, w, 4.0)


@pytest.mark.parametrize("rows,cols,k", [(20001, 128, 4), (9000, 64, 16), (3000, 1000, 20), (700, 9000, 40), (600, 33000, 64)])
def test_many_rows(r, rows, cols, k):
    """More rows than workgroups, in 64 bits on the GPU."""
    x, c, t, w = inputs_of(3, rows, cols, k, BF16)
    loss, dx = r.train_distill(x, c, t, 2.0, w, out=F32)
    log_q, log_p = torch.log_softmax(x.double() / 2, 1), torch.log_softmax(t.double() / 2, 1)
    ref = 4 * w.double() * (log_p.exp() * (log_p - log_q.gather(1, c))).sum(1)
    grad = 2 * w.double()[:, None] * log_q.exp().scatter_add(1, c, -log_p.exp())
    # arguments are below 20 and logarithms below 15: the bounds above with 4 * 20 + 100 + 8 and (4 * 20 + 200 + 16) * 2 * 35 roundings
    assert ((loss.double() - ref).abs() <= 4 * w * 21000 * U).all()
    big = log_q.exp().scatter_add(1, c, log_p.exp())
    assert ((dx.double() - grad).abs() <= 2 * w[:, None] * (400 * U * big + LEAST)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,k", [(140001, 64, 3), (140001, 128, 4), (66001, 61, 5), (66001, 125, 20), (66001, 250, 3), (33001, 507, 9), (16500, 1001, 33),
                                         (8300, 2043, 70), (8300, 4090, 5), (4200, 8191, 65), (2100, 16383, 128), (1100, 20007, 64), (600, 33001, 9)])
def test_rows_of_a_workgroup_after_its_first(r, rows, cols, k, dtype):
    """Rows are independent of each other: a call that gives each workgroup several has the bits of calls that give it one."""
    x, _, _, w = inputs_of(1, rows, cols, 1, dtype, pad=1)
    g = torch.Generator().manual_seed(2)
    c, t = torch.randint(-1, cols + 1, (rows, k), generator=g).cuda(), torch.randn(rows, k, generator=g).cuda()
    c[::3, k - 1] = c[::3, 0]       # classes that come twice in some rows
    loss, dx = r.train_distill(x, c, t, 2.0, w)
    per = rows // 5 + 1
    for at in range(0, rows, per):
        part = slice(at, at + per)
        loss2, dx2 = r.train_distill(x[part], c[part], t[part], 2.0, w[part])
        assert torch.equal(loss[part], loss2) and torch.equal(dx[part], dx2)


def test_gradient_against_differences(r):
    x, c, t, w = inputs_of(1, 3, 21, 5)
    _, dx = r.train_distill(x, c, t, 1.5, w, out=F32)
    vx, step = f64(x), 1e-5
    for i in np.ndindex(vx.shape):
        up, down = vx.copy(), vx.copy()
        up[i] += step
        down[i] -= step
        slope = (O.distill(up, c.cpu().numpy(), f64(t), 1.5, f64(w))[0].sum() - O.distill(down, c.cpu().numpy(), f64(t), 1.5, f64(w))[0].sum()) / (2 * step)
        assert abs(float(dx[i]) - slope) <= 1e-6       # fp32's parts in 10^7 of values below 3, and the step's square


def test_rows_without_anything_to_learn(r):
    nan = float("nan")
    for cols in (5, 70, 700, 5000):
        x, c, t, _ = inputs_of(2, 6, cols, 3)
        w = torch.ones(6, device="cuda")
        c[0], t[0] = torch.tensor([-1, cols, 1 << 40]), nan        # no entry given
        t[1] = -INF                                                # none above -inf
        x[2] = -INF                                                # no class left
        w[3], x[3], t[3] = 0.0, nan, nan                           # no weight
        for out in (F32, BF16):
            loss, dx = r.train_distill(x, c, t, 2.0, w, out=out)
            assert (loss[:4] == 0).all() and (dx[:4] == 0).all() and (loss[4:] > 0).all() and (dx[4:] != 0).any(1).all()


def test_infinities_and_nan(r):
    nan = float("nan")
    for cols in (6, 90, 3000):
        x, c, t, _ = inputs_of(4, 6, cols, 2)
        x[0, c[0, 1]] = -INF      # an entry of a class without probability
        x[1, 0] = nan
        x[2, cols - 1] = INF
        t[3, 1] = nan
        t[4, 0] = INF
        loss, dx = r.train_distill(x, c, t, out=F32)
        assert loss[0] == INF and torch.isfinite(dx[0]).all() and dx[0, c[0, 1]] < 0
        assert torch.isnan(loss[1:5]).all() and torch.isnan(dx[1]).all() and torch.isnan(dx[2]).all()
        assert torch.isnan(dx[3].gather(0, c[3])).all() and torch.isnan(dx[4].gather(0, c[4])).all()
        assert torch.isfinite(loss[5]) and torch.isfinite(dx[5]).all()


def test_masks_of_the_lowest_value(r):
    """Logits of the type's lowest value act as -inf beside others, and as any equal values among themselves."""
    for dtype in (F32, BF16):
        for temp in (0.25, 1.0, 3.0):
            x, c, t, _ = inputs_of(6, 4, 50, 3, dtype)
            off = torch.ones_like(x, dtype=torch.bool).scatter(1, c, False) & (torch.arange(50, device="cuda") % 2 == 0)
            low = torch.where(off, torch.finfo(dtype).min, x)
            for u, v in zip(r.train_distill(low, c, t, temp, out=F32), r.train_distill(torch.where(off, -INF, x), c, t, temp, out=F32)):
                assert torch.equal(u, v)
            low[:] = torch.finfo(dtype).min
            for u, v in zip(r.train_distill(low, c, t, temp, out=F32), r.train_distill(torch.zeros_like(x), c, t, temp, out=F32)):
                assert torch.equal(u, v)
            t[0] = torch.tensor([1.0, torch.finfo(F32).min, torch.finfo(F32).min])
            gone = t.clone()
            gone[0, 1:] = -INF
            for u, v in zip(r.train_distill(x, c, t, temp, out=F32), r.train_distill(x, c, gone, temp, out=F32)):
                assert torch.equal(u, v)


def test_what_lies_between_the_rows_stays(r):
    rows, cols, k = 37, 45, 4
    x, c, t, w = inputs_of(1, rows, cols, k)
    loss, dx = r.train_distill(x, c, t, 1.0, w, out=F32)
    for dtype, kind in ((F32, b.TYPE_FP32), (BF16, b.TYPE_BF16)):
        wide = torch.full((rows, cols + 3), 7.0, dtype=dtype, device="cuda")
        b.donerf_train_distill(r.h, (x.data_ptr(), cols, b.TYPE_FP32), (c.data_ptr(), k, b.TYPE_INT64), (t.data_ptr(), k, b.TYPE_FP32), w.data_ptr(), 1.0,
                               None, (wide.data_ptr(), cols + 3, kind), rows, cols, k)
        assert torch.equal(wide[:, :cols], dx.to(dtype)) and (wide[:, cols:] == 7).all()


def test_no_rows(r):
    loss, dx = r.train_distill(torch.empty(0, 5, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda"))
    assert loss.shape == (0,) and dx.shape == (0, 5)


def test_a_render_as_teacher(r):
    """A larger oracle's dumped classes and scores are entries as they are."""
    out = r.render(inputs.make_poses([0]), 24, 20, 4, debug=True)
    scores, bins = out["scores"].view(-1, 128), out["bins"].view(-1, 4)
    x = scores + torch.randn(scores.shape, generator=torch.Generator().manual_seed(1)).cuda()
    check(r, x, bins, scores.gather(1, bins.long()), None, 2.0, F32)


def test_refusals(r):
    x, c, t, w = inputs_of(1, 6, 20, 3)
    for call in (lambda: r.train_distill(x.half(), c, t), lambda: r.train_distill(x, c.float(), t), lambda: r.train_distill(x, c, t.double()),
                 lambda: r.train_distill(x, c[:5], t[:5]), lambda: r.train_distill(x, c, t[:, :2]), lambda: r.train_distill(x, c.cpu(), t),
                 lambda: r.train_distill(x, c, t, row_weight=w[:5]), lambda: r.train_distill(x, c, t, row_weight=w.double()),
                 lambda: r.train_distill(x, c[:, 0], t), lambda: r.train_distill(x.t(), c, t), lambda: r.train_distill(x, c, t, out=torch.float16)):
        with pytest.raises(ValueError):
            call()
    for temp in (0.0, -1.0, float("nan"), 1e9):
        with pytest.raises(b.DonerfError, match="temperature"):
            r.train_distill(x, c, t, temp)
    with pytest.raises(b.DonerfError, match="entries"):
        r.train_distill(x, c.repeat(1, 43), t.repeat(1, 43))
    with pytest.raises(b.DonerfError, match="dx overlaps"):
        b.donerf_train_distill(r.h, (x.data_ptr(), 20, b.TYPE_FP32), (c.data_ptr(), 3, b.TYPE_INT64), (t.data_ptr(), 3, b.TYPE_FP32), None, 1.0, None,
                               (x.data_ptr(), 20, b.TYPE_FP32), 6, 20, 3)
    with pytest.raises(b.DonerfError, match="loss overlaps"):
        b.donerf_train_distill(r.h, (x.data_ptr(), 20, b.TYPE_FP32), (c.data_ptr(), 3, b.TYPE_INT64), (t.data_ptr(), 3, b.TYPE_FP32), None, 1.0, t.data_ptr(),
                               None, 6, 20, 3)
    with torch.cuda.stream(torch.cuda.Stream()):
        with pytest.raises(ValueError, match="stream"):
            r.train_distill(x, c, t)


# ---- high temperatures: p and q are close to each other, and the loss, T^2 times a sum of their
# differences' squares, is as large as ever

def reference(x, classes, t, temp, weight):
    """(loss, dx, the bounds of both without a final rounding) of one row, in 80 bits: those of 64, times T^2, are themselves off by
    parts in a million."""
    x, t = x.astype(np.longdouble), t.astype(np.longdouble)
    given = (classes >= 0) & (classes < len(x))
    c, t = classes[given], t[given]
    un, tn = (x - x.max()) / temp, (t - t.max()) / temp
    e, f = np.exp(un), np.exp(tn)
    keep = f > 2.0 ** -126
    c, tn, f = c[keep], tn[keep], f[keep]
    sq, sp = e.sum(), f.sum()
    p, q = f / sp, e / sq
    delta = tn - un[c] - (np.log(sp) - np.log(sq))
    loss, grad = (p * delta).sum(), q.copy()
    np.add.at(grad, c, -p)
    # an argument is off by 3u (difference, 1/T and product), an exponential by 2u more, a sum by SUM
    _, first = np.unique(c, return_index=True)
    first = np.isin(np.arange(len(c)), first)
    rest = np.ones(len(x), bool)
    rest[c] = False
    au, at = np.where(np.isfinite(un), np.abs(un), 0), np.abs(tn)
    rel_q, rel_p = (e * (3 * U * au + 2 * U)).sum() / sq + SUM + 2 * U, (f * (3 * U * at + 2 * U)).sum() / sp + SUM + 2 * U
    # sp - sq: below 1 an expm1 is off by 3u and 2u of its argument at most; classes without an entry, and entries of a class that has
    # another, come as they are
    apart = (5 * U + SUM) * (at + au[c])[first].sum() + ((3 * U * at + 2 * U + SUM) * f)[~first].sum() + (e * (3 * U * au + 2 * U + SUM))[rest].sum()
    z = (sp - sq) / sq
    by_ratio = 2 * (apart / sq + abs(z) * (rel_q + 3 * U)) + 2 * U * abs(np.log1p(z))
    by_logs = rel_p + rel_q + 3 * U * (abs(np.log(sp)) + abs(np.log(sq)))
    of_log = by_ratio if abs(z) < 0.49 else by_logs if abs(z) > 0.51 else max(by_ratio, by_logs)
    ed = 3 * U * (at + au[c]) + 2 * U * (at + au[c] + abs(np.log(sp / sq))) + of_log
    ep, eq, ad = p * (rel_p + 3 * U * at + 4 * U), q * (rel_q + 3 * U * au + 4 * U), np.abs(delta)
    # e^-d - 1 + d is off by 10 roundings, and by its slope, below 1.7 |d|, times the error of d; further off it is the difference itself
    close, far = ad < 0.51, ad > 0.49
    of_terms = np.where(close, (ep + 12 * U * p) * ad ** 2 + p * (1.7 * ad * ed + ed ** 2), 0) + np.where(far, (ep + 3 * U * p) * (ad + 1) + p * ed + eq[c] + 2 * U * q[c], 0)
    of_grad = np.where(close, (ep + 12 * U * p) * 1.4 * ad + 1.7 * p * ed, 0) + np.where(far, ep + eq[c] + 2 * U * (p + q[c]), 0)
    terms = np.abs(p * delta + q[c] - p)
    more = (e[c][~first]).sum() / sq
    bl = of_terms.sum() + SUM * terms.sum() + eq[rest].sum() + SUM * (q[rest].sum() + more) + eq[c][~first].sum() + rel_q * (q[rest].sum() + more) + 4 * U * abs(loss)
    bd = np.where(rest, eq, 0)
    np.add.at(bd, c, of_grad + (0 if first.all() else ep + (len(c) + 4) * U * p))
    if not first.all():
        bd += eq
    w = abs(float(weight))
    return [np.asarray(v, np.float64) for v in (weight * temp ** 2 * loss, weight * temp * grad, w * temp ** 2 * bl, w * temp * (bd + 4 * U * np.abs(grad) + LEAST))]


def check_high(r, x, classes, t, temp, weight):
    vx, vc, vt, vw = f64(x), classes.cpu().numpy(), f64(t), f64(weight)
    for out in (F32, BF16):
        loss, dx = r.train_distill(x, classes, t, temp, weight, out=out)
        for i in range(len(vx)):
            ref_l, ref_d, bl, bd = reference(vx[i], vc[i], vt[i], temp, vw[i])
            assert abs(float(loss[i]) - ref_l) <= bl + U * abs(ref_l), (i, float(loss[i]), ref_l, bl)
            assert (np.abs(f64(dx[i]) - ref_d) <= bd + HALF[out] * (np.abs(ref_d) + bd)).all(), (i, np.abs(f64(dx[i]) - ref_d).max())
        again = r.train_distill(x, classes, t, temp, weight, out=out)
        assert torch.equal(loss, again[0]) and torch.equal(dx, again[1])


FULL = [(40, 1, 1), (30, 3, 3), (20, 8, 8), (20, 9, 9), (20, 24, 24), (20, 64, 64), (20, 61, 61), (12, 65, 65), (12, 128, 128), (9, 125, 125), (12, 100, 90),
        (9, 200, 128), (5, 283, 33), (4, 700, 128), (4, 1500, 50), (3, 3000, 128), (3, 7001, 7), (2, 16384, 128), (2, 20007, 64), (1, 32000, 9),
        (2, 40001, 128), (1, 65536, 3)]


@pytest.mark.parametrize("temp", [4.5, 64.0, 4096.0, 65536.0])
@pytest.mark.parametrize("rows,cols,k", FULL)
def test_high_temperatures(r, rows, cols, k, temp):
    for dtype in (F32, BF16):
        x, c, t, w = inputs_of(rows + cols, rows, cols, k, dtype, pad=1)
        check_high(r, x, c, t, temp, w)
        # all probability with the entries' classes: the others masked, by either value
        rest = torch.ones_like(x, dtype=torch.bool).scatter(1, c, False)
        for low in (-INF, torch.finfo(dtype).min):
            check_high(r, torch.where(rest, low, x), c, t, temp, w)
        x, c, t, w = inputs_of(rows + cols + 1, rows, cols, k, dtype, torch.int32, twice=True)
        check_high(r, x, c, t, temp, w)
        t[:, ::3] = torch.where(torch.arange(k, device="cuda")[::3] > 0, torch.finfo(F32).min, t[:, ::3])       # entries without probability
        check_high(r, x, c, t, temp, w)


@pytest.mark.parametrize("temp", [8.0, 4096.0])
def test_high_temperature_of_equal_and_near_logits(r, temp):
    """A student that has its teacher's logits has no loss and no gradient; one next to it a positive loss."""
    for cols in (5, 64, 100, 128):
        x, _, _, w = inputs_of(cols, 30, cols, 1)
        c = torch.stack([torch.randperm(cols, generator=torch.Generator().manual_seed(i)) for i in range(30)]).cuda()
        loss, dx = r.train_distill(x, c, x.gather(1, c), temp, w, out=F32)
        # sums of the same terms in two orders: delta is a rounding or two of their size
        size = f64(x.max(1).values - x.min(1).values) / temp
        assert (np.abs(f64(loss)) <= temp ** 2 * f64(w) * (SUM * size) ** 2).all() and (np.abs(f64(dx)).max(1) <= temp * f64(w) * SUM * size).all()
        loss, _ = r.train_distill(x, c, x.gather(1, c) * 1.01, temp, w)
        assert (loss > 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,k", [(140001, 64, 3), (140001, 128, 4), (66001, 61, 5), (66001, 125, 20), (66001, 250, 3), (33001, 507, 9), (16500, 1001, 33),
                                         (8300, 2043, 70), (8300, 4090, 5), (4200, 8191, 65), (2100, 16383, 128), (1100, 20007, 64), (600, 33001, 9)])
def test_rows_after_a_workgroups_first_at_high_temperatures(r, rows, cols, k, dtype):
    x, _, _, w = inputs_of(1, rows, cols, 1, dtype, pad=1)
    g = torch.Generator().manual_seed(2)
    c, t = torch.randint(-1, cols + 1, (rows, k), generator=g).cuda(), torch.randn(rows, k, generator=g).cuda()
    c[::3, k - 1] = c[::3, 0]
    w[::7] = 0
    loss, dx = r.train_distill(x, c, t, 32.0, w)
    per = rows // 5 + 1
    for at in range(0, rows, per):
        part = slice(at, at + per)
        loss2, dx2 = r.train_distill(x[part], c[part], t[part], 32.0, w[part])
        assert torch.equal(loss[part], loss2) and torch.equal(dx[part], dx2)
    only, none = r.train_distill(x, c, t, 32.0, w, need_dx=False)
    assert none is None and torch.equal(loss, only)


def test_edges_at_high_temperatures(r):
    nan = float("nan")
    for cols in (6, 90, 700, 3000, 40000):
        x, c, t, _ = inputs_of(4, 10, cols, 2)
        w = torch.ones(10, device="cuda")
        x[0, c[0, 1]] = -INF      # an entry of a class without probability
        x[1, 0] = nan
        x[2, cols - 1] = INF
        t[3, 1] = nan
        t[4, 0] = INF
        c[5], t[5] = torch.tensor([-1, cols]), nan
        t[6] = -INF
        x[7] = -INF
        w[8], x[8], t[8] = 0.0, nan, nan
        for out in (F32, BF16):
            loss, dx = r.train_distill(x, c, t, 1000.0, w, out=out)
            assert loss[0] == INF and torch.isfinite(dx[0]).all() and dx[0, c[0, 1]] < 0
            assert torch.isnan(loss[1:5]).all() and torch.isnan(dx[1]).all() and torch.isnan(dx[2]).all()
            assert torch.isnan(dx[3].gather(0, c[3])).all() and torch.isnan(dx[4].gather(0, c[4])).all()
            assert (loss[5:9] == 0).all() and (dx[5:9] == 0).all()
            assert loss[9] > 0 and torch.isfinite(dx[9]).all() and (dx[9] != 0).any()
