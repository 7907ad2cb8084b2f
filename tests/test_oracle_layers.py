"""The numpy oracle of the layer operators against values worked out by hand,
against E4M3 as the networks' oracle has it, and against differences."""
import numpy as np
import pytest

from oracle import layers_oracle as L


def one_block(vals, fmt):
    x = np.zeros((1, 32))
    x[0, :len(vals)] = vals
    c, s = L.quantize(x, fmt)
    return L.values(c, s, 32, fmt)[0, :len(vals)], int(s[0, 0])


def test_mxfp4_by_hand():
    # largest 6: scale 1; ties go to the even code
    v, s = one_block([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5.1, 0.26, -0.2], "mxfp4")
    assert s == 127
    assert v.tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -6, 0.5, 0]
    # just above 6 the scale doubles, at 3 it halves
    assert one_block([6.01, 1.0], "mxfp4") == (pytest.approx([6.0, 1.0]), 128)
    assert one_block([3.0], "mxfp4")[1] == 126
    assert one_block([0.0], "mxfp4") == (pytest.approx([0.0]), 0)


def test_mxfp8_by_hand():
    v, s = one_block([448, 2.0 ** -9, 2.0 ** -30, 17, 19, -21, 0], "mxfp8")
    assert s == 127
    # 17 and 19 lie between 16 and 18, 18 and 20; a tie goes to the even code
    assert v.tolist() == [448, 2.0 ** -9, 2.0 ** -9, 16, 20, -20, 0]
    assert one_block([449.0], "mxfp8")[1] == 128 and one_block([224.0], "mxfp8")[1] == 126


def test_not_finite():
    x = np.ones((1, 64))
    x[0, 3], x[0, 40] = np.nan, np.inf
    c, s = L.quantize(x, "mxfp4")
    assert s.tolist() == [[255, 255]] and np.isnan(L.values(c, s, 64, "mxfp4")).all()
    c, s = L.quantize(x, "mxfp8")
    v = L.values(c, s, 64, "mxfp8")
    assert np.isnan(v[0, [3, 40]]).all() and np.isnan(v).sum() == 2 and (np.delete(v[0], [3, 40]) == 1).all()


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
def test_packing_and_rounding(fmt):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((20, 75)) * np.exp2(rng.integers(-140, 100, (20, 1)).astype(float))
    c, s = L.quantize(x, fmt)
    assert np.array_equal(L.unpack(L.pack(c, fmt), fmt), c)
    v = L.values(c, s, 75, fmt)
    assert (np.abs(v - x) <= L.half_step(x, s, fmt)).all()
    # what a format holds is held exactly
    c2, s2 = L.quantize(v, fmt)
    assert np.array_equal(L.values(c2, s2, 75, fmt), v)


def test_e4m3_as_the_networks_oracle_has_it():
    from oracle import donerf_oracle as O
    x = np.concatenate([np.random.default_rng(5).uniform(2.0 ** -9, 448, 999), L.GRID["mxfp8"][1:], [448.0]])
    c, s = L.quantize(np.stack([x, np.full(x.shape, 448.0)], 1), "mxfp8")     # the 448 makes the scale 1
    assert (s == 127).all()
    assert np.array_equal(L.values(c, s, 1, "mxfp8")[:, 0], np.asarray(O.round_e4m3(x), np.float64))


def test_gradients_against_differences():
    rng = np.random.default_rng(4)
    u, w, b, dz = (rng.standard_normal(s) for s in ((5, 7), (3, 7), (3,), (5, 3)))
    loss = lambda u, w, b: float((dz * L.linear(np.maximum(u, 0), w, b)).sum())
    dx, dw, db = L.backward(dz, np.maximum(u, 0), w, relu=True)
    for i, (t, g) in enumerate(((u, dx), (w, dw), (b, db))):
        for at in np.ndindex(t.shape):
            d = np.zeros(t.shape)
            d[at] = 1e-6
            args = [u, w, b]
            hi, lo = [*args], [*args]
            hi[i], lo[i] = t + d, t - d
            # the loss is piecewise linear: differences are exact but for rounding
            assert abs((loss(*hi) - loss(*lo)) / 2e-6 - g[at]) < 1e-7
