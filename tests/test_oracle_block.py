"""Pins of oracle/block_oracle.py: against other ways of writing the same functions, and gradients against differences."""
import numpy as np
import pytest

from oracle import block_oracle as bo

PAIRS, THETA = (22, 21, 21), (10000.0, 10000.0, 500.0)


def _rng(*seed):
    return np.random.default_rng(seed)


@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
def test_rotation_is_a_complex_factor_and_relative(pairing):
    r = _rng(1)
    x, y = r.standard_normal((2, 1, 1, 1, 128))
    pos = np.array([[[7, -3, 100]]])
    lo, hi = bo.pair_channels(pairing)
    ang = bo.angles(pos, PAIRS, THETA)
    z = (x[..., lo] + 1j * x[..., hi]) * np.exp(1j * ang)
    got = bo.rope_fwd(x, ang, pairing)
    assert np.allclose(got[..., lo], z.real) and np.allclose(got[..., hi], z.imag)
    # a product of two turned rows depends on the difference of their positions alone
    shift = np.array([[[1000, 5, -40]]])
    a = (bo.rope_fwd(x, bo.angles(pos, PAIRS, THETA), pairing) * bo.rope_fwd(y, bo.angles(pos * 0, PAIRS, THETA), pairing)).sum()
    b = (bo.rope_fwd(x, bo.angles(pos + shift, PAIRS, THETA), pairing) * bo.rope_fwd(y, bo.angles(shift, PAIRS, THETA), pairing)).sum()
    assert abs(a - b) < 1e-10
    assert np.allclose(ang[0, 0, [0, 22, 43]], [7 - 2 * np.pi, -3, 100 - 15 * 2 * np.pi])   # (each axis starts at one radian a step)
    assert np.allclose(np.exp(1j * ang[0, 0, [21, 42, 63]]), np.exp(1j * np.array([7, -3, 100]) *
                                                                    np.array([1e4 ** (-21 / 22), 1e4 ** (-20 / 21), 500 ** (-20 / 21)])))


def _difference(f, x, direction, step=1e-5):
    return (f(x + step * direction) - f(x - step * direction)) / (2 * step)


@pytest.mark.parametrize("norm", ["none", "head", "token"])
@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
def test_rope_gradients_against_differences(norm, pairing):
    r = _rng(2)
    x, dy, dirx = r.standard_normal((3, 2, 3, 4, 128))
    w = 1 + 0.2 * r.standard_normal(128 if norm == "head" else 3 * 128)
    dirw = r.standard_normal(w.shape)
    ang = bo.angles(r.integers(-50, 50, (2, 4, 3)), PAIRS, THETA)
    dx, dw, scale = bo.rope_bwd(dy, x, ang, pairing, w, norm)
    loss = lambda x_, w_: (bo.rope_fwd(x_, ang, pairing, w_, norm) * dy).sum()
    assert _difference(lambda t: loss(t, w), x, dirx) == pytest.approx((dx * dirx).sum(), rel=1e-7, abs=1e-7)
    assert (scale >= np.abs(dx) * (1 - 1e-12)).all()
    if norm != "none":
        assert _difference(lambda t: loss(x, t), w, dirw) == pytest.approx((dw * dirw).sum(), rel=1e-7, abs=1e-7)


def test_norm_gradients_against_differences():
    r = _rng(3)
    h, dy, dh, dirh = r.standard_normal((4, 5, 24))
    w, dirw = 1 + 0.2 * r.standard_normal((2, 24))
    dx, dw, scale = bo.norm_bwd(dy, h, w, dh, 1e-3)
    loss = lambda h_, w_: (bo.norm_fwd(h_, w_, 1e-3) * dy).sum() + (h_ * dh).sum()
    assert _difference(lambda t: loss(t, w), h, dirh) == pytest.approx((dx * dirh).sum(), rel=1e-7, abs=1e-7)
    assert _difference(lambda t: loss(h, t), w, dirw) == pytest.approx((dw * dirw).sum(), rel=1e-7, abs=1e-7)
    assert (scale >= np.abs(dx) * (1 - 1e-12)).all()
    assert np.allclose((bo.norm_fwd(h, None, 0.0) ** 2).mean(1), 1.0)


@pytest.mark.parametrize("lens", [None, (7, 0), (3, 7)])
def test_cross_attention_by_scalars_and_gradients_against_differences(lens):
    r = _rng(4)
    q, do, dirq = r.standard_normal((3, 2, 4, 3, 128))
    k, v, dirk, dirv = r.standard_normal((4, 2, 2, 7, 128))
    out, lse = bo.xattn_fwd(q, k, v, lens)
    for b in range(2):
        n = 7 if lens is None else lens[b]
        for h in range(4):
            for i in range(3):
                w = [np.exp(float(q[b, h, i] @ k[b, h // 2, t]) / np.sqrt(128.0)) for t in range(n)]
                want = sum((w[t] * v[b, h // 2, t] for t in range(n)), np.zeros(128)) / (sum(w) or 1.0)
                assert np.allclose(out[b, h, i], want)
                assert lse[b, h, i] == (pytest.approx(np.log(sum(w))) if n else -np.inf)
    dq, dk, dv = bo.xattn_bwd(q, k, v, do, lens)
    loss = lambda q_, k_, v_: (bo.xattn_fwd(q_, k_, v_, lens)[0] * do).sum()
    assert _difference(lambda t: loss(t, k, v), q, dirq) == pytest.approx((dq * dirq).sum(), rel=1e-6, abs=1e-6)
    assert _difference(lambda t: loss(q, t, v), k, dirk) == pytest.approx((dk * dirk).sum(), rel=1e-6, abs=1e-6)
    assert _difference(lambda t: loss(q, k, t), v, dirv) == pytest.approx((dv * dirv).sum(), rel=1e-6, abs=1e-6)
