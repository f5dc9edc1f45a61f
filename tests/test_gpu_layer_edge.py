"""The layer norm on the GPU where rounding the mean of a row would show: rows that are constant, or constant but for a feature or a few.

Tolerances, of n = ((h - p) - c) r with p the bf16 number next to the mean, c the rest of the mean and s^2 the variance.  All features of a row
are bf16 numbers within a factor of four here: their sum, of at most 2^14 numbers of 10 bits, is exact in fp32, and so is h - p; c, at most s (no
feature lies between the two bf16 numbers around the mean), is off by its subtraction's rounding, that of 1 / K and of the product: 2^-22 s.  The
variance is the mean of (h - p)^2, at most 2 s^2, less c^2.  Sums are at most 54 additions deep (32 of a thread, then 64 threads in
pairs, then up to 16 wavefronts), each of 2^-24, so it is off by less than 2^-18 2 s^2 + 2^-21 s^2 < 2^-16 s^2, r by 2^-17 of itself and n
by 2^-22 + 2^-17 |n|, a few 2^-23 of its terms aside: below N = 2^-15 (1 + |n|).  Of a constant row p is the feature itself and c
zero, so n is zero: exactly.  A result in bf16 is off by half a step more, 2^-8 of its size.
Backward, with g = dy: r g and r mean(g) are off by 2^-15 of their sizes, n mean(g n) by N for each of its two n; sums over rows add up
N |dy|, and 2^-24 of their sizes for each of a few rows."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mo
from paper_2512_16093_amd import binding as sla

pytestmark = pytest.mark.gpu

HALF, N = 2.0 ** -8, 2.0 ** -15
VALUES = [3.0, 1000.0, -4000.0, 20608.0, 1.0, 0.3, -250.0, 1e17, 1e-30]      # (of a row, rounded to bf16)
WIDTHS = [8, 72, 520, 1000, 1304, 1528, 2048, 2056, 3080, 5128, 6008, 7000, 8200, 11000, 16376]


def _np(t):
    return t.detach().double().cpu().numpy()


def _cuda(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16().cuda()


def _rows(K, M=len(VALUES)):
    return _cuda(np.resize(np.array(VALUES), M)[:, None] * np.ones((1, K)))


def _vectors(r, K):
    six = torch.from_numpy((0.4 * r.standard_normal((1, 6, K))).astype(np.float32)).cuda()
    return dict(w=_cuda(1 + 0.2 * r.standard_normal(K)), bias=_cuda(0.3 * r.standard_normal(K)), scale=six[:, 1], shift=six[:, 0])


@pytest.mark.parametrize("K", WIDTHS)
def test_constant_rows(K):
    r = np.random.default_rng(K)
    x, v = _rows(K), _vectors(r, K)
    assert (sla.norm_layer_fwd(x)[0] == 0).all()
    # what is left is the bias, scaled and shifted: the same bits in every row
    y = sla.norm_layer_fwd(x, **v)[0]
    up, b, t = 1 + _np(v["scale"]), _np(v["bias"])[None], _np(v["shift"])
    assert (np.abs(_np(y) - (b * up + t)) <= HALF * np.abs(b * up + t) + 2.0 ** -22 * (np.abs(b) * (1 + np.abs(up)) + np.abs(t))).all()
    assert (y == y[:1]).all()
    # a gate and a residual that leave the stored stream constant
    one = torch.ones((1, K), device="cuda")
    y2, h = sla.norm_layer_fwd(torch.zeros_like(x), res=x, gate=one, **v)
    assert torch.equal(h, x) and torch.equal(y2, y)
    # backward: n is zero, so weights and scales have no gradient from it and dx = r (g - mean(g))
    dy = _cuda(r.standard_normal(x.shape))
    for up in (dy, torch.ones_like(dy)):
        got = sla.norm_layer_bwd(up, x, w=v["w"], bias=torch.zeros_like(v["bias"]), scale=v["scale"])
        assert (got.dw == 0).all() and (got.dscale == 0).all()
        g = _np(up)
        want = (g - g.mean(1, keepdims=True)) * 1e3
        size = 1e3 * (np.abs(g) + np.abs(g).mean(1, keepdims=True))
        dx = sla.norm_layer_bwd(up, x, want_vectors=False).dx
        assert (np.abs(_np(dx) - want) <= HALF * np.abs(want) + N * size).all()


@pytest.mark.parametrize("M,K", [(4099, 2056), (4097, 1000), (4096, 8200)])
def test_constant_rows_two_at_a_time_and_into_codes(M, K):
    x, v = _rows(K, M), _vectors(np.random.default_rng(K), K)
    y = sla.norm_layer_fwd(x, **v)[0]
    assert (y == y[:1]).all()
    assert (sla.norm_layer_fwd(x)[0] == 0).all()
    q, _ = sla.mxfp4_norm_quantize(x, **v)
    assert all(torch.equal(a, b) for a, b in zip(sla.mxfp4_unpack(q, M, K), sla.mxfp4_unpack(sla.mxfp4_quantize(y), M, K)))
    assert (sla.mxfp4_unpack(sla.mxfp4_norm_quantize(x)[0], M, K)[0] & 0x77 == 0).all()      # (zeros of either sign)


def _nearly(K):
    """Rows of one bf16 number, with its neighbour at one feature, at three, at a third of them; and up and down in turn."""
    of = _np(_cuda(np.array([1000.0, -4000.0, 20608.0, 1.0, 0.3])))
    x = np.tile(np.repeat(of, 4)[:, None], (1, K))
    step = np.ldexp(1.0, np.frexp(x)[1] - 8)                         # (of 8 significant bits)
    x[0::4, K // 2] += step[0::4, 0]
    x[1::4, [0, 3, K - 1]] += step[1::4, :1]
    x[2::4, ::3] += step[2::4, :1]
    x[3::4, 1::2] += step[3::4, :1]
    x[3::4, ::2] -= step[3::4, :1] * (np.abs(x[3::4, :1]) != 1.0)     # (below a power of two the steps are half as long)
    t = _cuda(x)
    assert (_np(t) == x).all()
    return t


@pytest.mark.parametrize("K", WIDTHS)
def test_nearly_constant_rows(K):
    r = np.random.default_rng(K + 1)
    x = _nearly(K)
    h = _np(x)
    n, f, _ = mo.layer_rows(h, 1e-6)
    off = N * (1 + np.abs(n))
    assert (np.abs(_np(sla.norm_layer_fwd(x)[0]) - n) <= HALF * np.abs(n) + off).all()
    big = x.repeat(206, 1)                                           # (4120 rows: two at a time where a vector is shared)
    got = sla.norm_layer_fwd(big, shift=torch.zeros((1, K), device="cuda"))[0]
    assert (got.view(206, *x.shape) == sla.norm_layer_fwd(x)[0]).all()
    for dy in (_cuda(r.standard_normal(x.shape)), _cuda(np.where(h == h[:, 1:2], 1.0, -2.0))):
        g = _np(dy)
        mean = lambda t: t.mean(1, keepdims=True)
        got = sla.norm_layer_bwd(dy, x, w=torch.ones(K, dtype=torch.bfloat16, device="cuda"))
        assert (np.abs(_np(got.dw) - (g * n).sum(0)) <= (np.abs(g) * (off + x.shape[0] * 2.0 ** -24 * np.abs(n))).sum(0)).all()
        want = f * (g - mean(g) - n * mean(g * n))
        a, m = np.abs(n), np.abs(g)
        # (the two products' own roundings are a few 2^-23 of their sizes, and the mean of g n is 54 additions deep: 2^-18 of its terms' sizes)
        fp32 = f * (N * (m + mean(m)) + off * mean(m * a) + a * mean(m * off) + 2.0 ** -15 * a * mean(m * a))
        assert (np.abs(_np(got.dx) - want) <= HALF * np.abs(want) + fp32).all()


def test_the_most_rows_with_a_vector_each():
    """2^22 rows in as many samples (of one vector, at stride 0) by the widest teams: 2^32 threads, more than a launch has in a row."""
    M, K = 1 << 22, 12296
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 4.2 * M * K:
        pytest.skip("two tensors of 103 GB do not fit beside what is on the card")
    r = np.random.default_rng(3)
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    few, places = _cuda(2 * r.standard_normal((4, K))), (0, M // 2 - 2, M - 4)
    for at in places:
        x[at:at + 4] = few
    v = {k: torch.from_numpy(r.standard_normal((1, K)).astype(np.float32)).cuda() for k in ("scale", "shift")}
    wide = {k: t.expand(M, K) for k, t in v.items()}
    want, rest = sla.norm_layer_fwd(few, **v)[0], v["shift"].bfloat16()[0]
    q, _ = sla.mxfp4_norm_quantize(x, **wide)
    codes, exps = sla.mxfp4_unpack(q, M, K)
    del q
    want_codes, want_exps = sla.mxfp4_unpack(sla.mxfp4_quantize(want), 4, K)
    rest_codes, rest_exps = sla.mxfp4_unpack(sla.mxfp4_quantize(rest[None]), 1, K)
    for at in places:
        assert torch.equal(codes[at:at + 4], want_codes) and torch.equal(exps[at:at + 4], want_exps)
    for at in (4, M // 2 + 2, M - 5):
        assert torch.equal(codes[at], rest_codes[0]) and torch.equal(exps[at], rest_exps[0])
    del codes, exps
    torch.cuda.empty_cache()
    y = torch.zeros_like(x)
    sla.norm_layer_fwd(x, **wide, out=y)
    for at in places:
        assert torch.equal(y[at:at + 4], want)
    for at in (4, M // 2 + 2, M - 5):
        assert torch.equal(y[at], rest)
    del x, y
    torch.cuda.empty_cache()
