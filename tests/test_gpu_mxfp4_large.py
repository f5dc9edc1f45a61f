"""The 4-bit layers on the GPU at their largest: objects and results beyond 2^32 bytes, tensors that exceed the caches, the widest
weights.  Some rows or columns of each call are checked; tolerances as in test_gpu_mxfp4.py."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mo
from paper_2512_16093_amd import binding as sla
from test_gpu_mxfp4 import _check, _np

pytestmark = pytest.mark.gpu


def _rand(seed, shape, amp=1.0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.bfloat16).mul_(amp)


def _some(M, n=60):
    return sorted({0, 1, M // 2, M - 2, M - 1, *np.random.default_rng(M).integers(0, M, n).tolist()})


def _held(x):
    return mo.dequantize(*mo.quantize(_np(x)))


@pytest.mark.parametrize("R,K", [(1200003, 64), (140001, 1000), (30001, 5120), (8209, 16384), (1100001, 8200)])
def test_there_and_back_past_the_caches(R, K):
    """The last one: the object itself has more than 2^32 bytes."""
    x = _rand(R, (R, K))
    nbytes = sla.mxfp4_bytes(R, K)
    around = torch.full((nbytes + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    q = sla.mxfp4_quantize(x, around[:nbytes])
    assert (around[nbytes:] == 0xA5).all()
    out = torch.full((R + 2, K), 7.0, dtype=torch.bfloat16, device="cuda")
    sla.mxfp4_dequantize(q, R, K, out[:R])
    assert (out[R:] == 7).all()
    at = _some(R)
    assert (_np(out[at]) == _held(x[at])).all()
    # every other row against a call of its own rows' tiles (the same rounding at another place)
    few = x[R - 4099:].contiguous()
    assert torch.equal(sla.mxfp4_dequantize(sla.mxfp4_quantize(few), 4099, K), out[R - 4099:R])


@pytest.mark.parametrize("M,N,K", [(1100001, 2056, 8200), (1100003, 2056, 264), (530001, 4104, 520), (300001, 264, 32776)])
def test_layers_of_very_many_tokens(M, N, K):
    """Results (the last: activations) beyond 2^32 bytes: walked tiles and wide ones, with the norm of the rows where it is that narrow."""
    x, w, bias = _rand(M, (M, K), 2.0), _rand(N, (N, K), K ** -0.5), _rand(3, N)
    wq = sla.mxfp4_quantize(w)
    out = torch.full((M + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
    sla.mxfp4_linear_fwd(x, wq, N, bias=bias, out=out[:M])
    assert (out[M:] == 7).all()
    at = _some(M)
    a, b = _held(x[at]), _np(sla.mxfp4_dequantize(wq, N, K))
    _check(out[at], a @ b.T + _np(bias), np.abs(a) @ np.abs(b).T + np.abs(_np(bias)), K)
    # the rows behind 2^32 bytes against a call of their own
    few = x[M - 3000:].contiguous()
    y = sla.mxfp4_linear_fwd(few, wq, N, bias=bias)
    # (each rounded to bf16, of sums in another order; a sum's sizes are at most the product of the lengths of its row and column)
    length = lambda q, R: sla.mxfp4_dequantize(q, R, K).float().norm(dim=1).double()
    size = torch.outer(length(sla.mxfp4_quantize(few), 3000), length(wq, N)) + bias.double().abs()
    fp32 = 2 * (7 * -(-K // 64) + 9) * 2.0 ** -23 * size
    assert bool(((y.double() - out[M - 3000:M].double()).abs() <= 2.0 ** -7 * (y.double().abs() + fp32) + fp32).all())


@pytest.mark.parametrize("M,N,K", [(1, 65536, 65536), (20, 65536, 40000), (130, 65528, 65528), (300, 65536, 4096), (4500, 65536, 1024), (70, 520, 65536), (2000, 264, 65536)])
def test_the_widest_weights(M, N, K):
    """The object of the first weight has more than 2^31 bytes."""
    x, w = _rand(M, (M, K)), _rand(N + 1, (N, K), K ** -0.5)
    wq = sla.mxfp4_quantize(w)
    out = torch.full((M + 1, N), 7.0, dtype=torch.bfloat16, device="cuda")
    sla.mxfp4_linear_fwd(x, wq, N, out=out[:M])
    assert (out[M] == 7).all()
    rows, cols = _some(M, 20) if M > 4 else list(range(M)), _some(N)
    a, b = _held(x[rows]), _held(w[cols])
    _check(out[rows][:, cols], a @ b.T, np.abs(a) @ np.abs(b).T, K)


def test_a_norm_into_an_object_beyond_32_bits():
    M, K = 1100001, 8200
    x = _rand(1, (M, K), 2.0)
    q, h = sla.mxfp4_norm_quantize(x)
    assert h is x and q.numel() > 2 ** 32
    back = sla.mxfp4_dequantize(q, M, K)
    del q
    for part in (slice(0, 5000), slice(M - 5000, M)):
        y = sla.norm_layer_fwd(x[part].contiguous())[0]
        assert torch.equal(back[part], sla.mxfp4_dequantize(sla.mxfp4_quantize(y), 5000, K))
