"""Pins of oracle/mx_oracle.py: the format's own values, ties and ends, other ways of writing the same functions, and gradients
against differences."""
import numpy as np
import pytest

from oracle import mx_oracle as mo


def _rng(*seed):
    return np.random.default_rng(seed)


def test_every_value_of_the_format_comes_back():
    for e in (-126, -7, 0, 1, 120):
        row = np.concatenate((mo.VALUES, -mo.VALUES, mo.VALUES, -mo.VALUES))[None] * 2.0 ** e
        codes, exps = mo.quantize(row)
        assert exps.tolist() == [[e + 127]] and (mo.dequantize(codes, exps) == row).all()
        assert codes[0, :16].tolist() == list(range(16))


def test_ties_ends_and_blocks_that_hold_no_number():
    row = np.zeros((1, 40))
    row[0, :16] = [6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 7.9, .2500001, .7499999, 1.2500001, 4.9999, -5, -.25, -1.75]
    codes, exps = mo.quantize(row)
    assert (codes[0, :16] & 7).tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 7, 1, 1, 3, 6, 6, 0, 4] and exps.tolist() == [[127, 1]]
    for bad in (np.inf, -np.inf, np.nan):
        row[0, 35] = bad
        codes, exps = mo.quantize(row)
        assert exps.tolist() == [[127, 255]] and not codes[0, 32:].any() and np.isnan(mo.dequantize(codes, exps)[0, 32:]).all()
    # the smallest exponent: what is below it is rounded to multiples of 2^-127
    assert mo.quantize(np.full((1, 32), 2.0 ** -127))[1][0, 0] == 1
    assert (mo.dequantize(*mo.quantize(np.full((1, 32), 2.0 ** -127))) == 2.0 ** -127).all()
    assert (mo.dequantize(*mo.quantize(np.full((1, 32), 2.0 ** -129))) == 0).all()


def test_rounding_is_to_the_nearest_and_plain_rows_come_back():
    x = _rng(1).standard_normal((50, 104)) * 10.0 ** _rng(2).integers(-8, 8, (50, 1))
    codes, exps = mo.quantize(x)
    v = mo.dequantize(codes, exps)
    unit = np.repeat(2.0 ** (exps.astype(float) - 127), 32, 1)[:, :104]
    a = np.abs(x) / unit
    half = np.where(a < 2, 0.25, np.where(a < 4, 0.5, 1.0))
    assert (np.abs(v - x) / unit <= np.where(a > 6, 2.0, half)).all() and a.max() < 8 and (a.reshape(50, -1).max(1) >= 4).all()
    assert (mo.codes_of(mo.plain(codes)) == codes).all()


def _difference(f, x, direction, step=1e-6):
    return (f(x + step * direction) - f(x - step * direction)) / (2 * step)


@pytest.mark.parametrize("samples", [1, 3])
def test_layer_gradients_against_differences(samples):
    r = _rng(3, samples)
    M, K = 6, 24
    x, res, dy, up = r.standard_normal((4, M, K))
    w, b = 1 + 0.2 * r.standard_normal(K), r.standard_normal(K)
    gate, scale, shift = 0.5 * r.standard_normal((3, samples, K))
    rep = lambda v: np.repeat(v, M // samples, 0)

    def loss(x=x, res=res, w=w, b=b, gate=gate, scale=scale, shift=shift):
        h = x + rep(gate) * res
        return (mo.layer_fwd(h, w, b, scale, shift, 1e-5)[0] * dy).sum() + (h * up).sum()
    got = mo.layer_bwd(dy, x + rep(gate) * res, w, b, up, res, gate, scale, 1e-5, samples)
    for name, at, grad in (("x", x, "dx"), ("res", res, "dres"), ("w", w, "dw"), ("b", b, "dbias"), ("gate", gate, "dgate"),
                           ("scale", scale, "dscale"), ("shift", shift, "dshift")):
        d = r.standard_normal(at.shape)
        assert _difference(lambda t: loss(**{name: t}), at, d) == pytest.approx((got[grad][0] * d).sum(), rel=1e-6, abs=1e-7), name
        assert (got[grad][1] >= np.abs(got[grad][0]) * (1 - 1e-12)).all(), name


def test_layer_norm_without_vectors():
    h = _rng(4).standard_normal((5, 40)) + 3
    y, size = mo.layer_fwd(h, None, None, None, None, 0.0)
    assert np.allclose(y.mean(1), 0) and np.allclose(y.std(1), 1) and (size >= np.abs(y)).all()
