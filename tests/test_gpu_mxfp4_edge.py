"""The 4-bit layers on the GPU at the edges of what they take, one call at least of every kernel of the product: objects whose rows behind the last
hold 0xff, activations, weights and biases that are no finite numbers, exponents from one end to the other.

Tolerances as in test_gpu_mxfp4.py; everything else is bit for bit."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mo
from paper_2512_16093_amd import binding as sla
from test_gpu_mxfp4 import HALF, _np, _product

pytestmark = pytest.mark.gpu

KERNELS = [  # tokens straight from bf16 (4 and 8 wavefronts), split by 4 and 8, of 2 x 1 and 2 x 2 tiles; square of 4 and 3 stages; wide by their
    # number and by the contraction's length; walked by their number and by the length
    (3, 40, 264), (2, 72, 5128), (32, 256, 1536), (31, 136, 8200), (40, 264, 1032), (600, 1040, 512),
    (1000, 1032, 400), (4100, 2056, 776), (5000, 4104, 400), (2300, 2056, 2312), (8193, 8192, 1032), (5000, 5128, 2056),
]


def _bf16(seed, shape, amp=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16).mul_(amp)


def _poisoned(R, K):
    return torch.full((sla.mxfp4_bytes(R, K),), 0xFF, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("M,N,K", KERNELS)
def test_what_is_no_finite_number_stays_by_itself(M, N, K):
    x, w, bias = _bf16(M, (M, K)), _bf16(N, (N, K), K ** -0.5), _bf16(K, N)
    clean = sla.mxfp4_linear_fwd(x, sla.mxfp4_quantize(w), N, bias=bias)
    assert torch.isfinite(clean).all()
    x2, w2, b2 = x.clone(), w.clone(), bias.clone()
    x2[M // 2, K - 1], x2[M - 1, 0] = float("nan"), float("inf")
    w2[N - 1, 0] = float("inf")
    b2[1], b2[N // 2], b2[N - 2] = float("inf"), float("-inf"), float("nan")
    rows, cols = torch.ones(M, dtype=torch.bool, device="cuda"), torch.ones(N, dtype=torch.bool, device="cuda")
    rows[[M // 2, M - 1]] = False
    cols[[1, N // 2, N - 2, N - 1]] = False
    wq = sla.mxfp4_quantize(w2, _poisoned(N, K))
    y = sla.mxfp4_linear_fwd(x2, wq, N, bias=b2, workspace=_poisoned(M, K))
    g = sla.mxfp4_gemm_fwd(sla.mxfp4_quantize(x2, _poisoned(M, K)), wq, M, N, K, bias=b2)
    for got in (y, g):
        assert torch.isnan(got[~rows]).all() and torch.isnan(got[:, [N - 2, N - 1]]).all()
        assert (got[rows, 1] == float("inf")).all() and (got[rows, N // 2] == float("-inf")).all()
    assert torch.equal(y[rows][:, cols], clean[rows][:, cols])
    want = sla.mxfp4_gemm_fwd(sla.mxfp4_quantize(x), sla.mxfp4_quantize(w), M, N, K, bias=bias)
    assert torch.equal(g[rows][:, cols], want[rows][:, cols])


@pytest.mark.parametrize("M,N,K", KERNELS)
def test_rows_of_zeros_are_the_bias(M, N, K):
    """Every finite bf16 number as a bias, the subnormal ones among them: N after N of them."""
    w = sla.mxfp4_quantize(_bf16(N, (N, K), K ** -0.5))
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    bits = np.arange(0x7F80, dtype=np.uint16)
    bits = np.concatenate((bits, bits | 0x8000))
    bits = np.resize(bits, -(-len(bits) // N) * N).reshape(-1, N)
    few = bits if len(bits) <= 16 else bits[np.linspace(0, len(bits) - 1, 16).astype(int)]
    for b in few:
        bias = torch.from_numpy(b.view(np.int16).copy()).view(torch.bfloat16).cuda()
        assert (sla.mxfp4_linear_fwd(x, w, N, bias=bias) == bias).all()


@pytest.mark.parametrize("M,N,K", [(32, 256, 256), (255, 256, 256), (40, 264, 520), (1000, 1032, 512), (4100, 2056, 776), (5000, 4104, 400), (8415, 8192, 1024)])
def test_every_exponent_of_activations_with_every_one_of_weights(M, N, K):
    """Rows of one exponent each, 0 to 254 on both sides: wherever result and terms are normal fp32 numbers they are the product, down to
    2^-127 from one side and up to 2^127 from the other."""
    r = np.random.default_rng([M, N, K])
    objects = []
    for R in (M, N):
        e = (np.arange(R) * (1 if R >= 255 else 8) % 255).astype(np.uint8)
        codes = r.integers(0, 16, (R, K)).astype(np.uint8)
        objects.append(sla.mxfp4_pack(torch.from_numpy(mo.plain(codes)).cuda(), torch.from_numpy(np.repeat(e[:, None], -(-K // 32), 1)).cuda()))
    y = _np(sla.mxfp4_gemm_fwd(*objects, M, N, K))
    want, size = _product(*objects, M, N, K, None)
    within = size < 3.3e38
    assert within.any(1).all() and within.any(0).all()
    bad = within & ~(np.abs(y - want) <= HALF * np.abs(want) + (7 * -(-K // 64) + 9) * 2.0 ** -23 * size + 1e-37)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4])
    # far below fp32's range nothing is left, far above it no finite number
    assert (np.abs(y[size < 1e-46]) == 0).all()
    assert not np.isfinite(y[np.abs(want) > 1e39]).any()


@pytest.mark.parametrize("M,N,K", KERNELS + [(1100, 1304, 1800), (3000, 1800, 520), (2100, 2184, 136), (2300, 2056, 1536), (33000, 520, 520), (65600, 1032, 1024), (66000, 776, 1280), (20000, 5128, 2568)])
def test_counted_copy_waits_agree_with_full_waits(M, N, K):
    """The kernels of the larger products wait for their copies by hand-counted `vmcnt` values; a second build of the library
    (-DSLA_FULL_WAITS) waits for every copy each time.  The two agree bit for bit, in calls that follow one another at once."""
    import ctypes
    import os
    from paper_2512_16093_amd import build
    assert os.path.exists(build.LIB_FULL_WAITS), "run python -m paper_2512_16093_amd.build"
    full = ctypes.CDLL(build.LIB_FULL_WAITS).mxfp4_gemm_fwd
    full.restype, full.argtypes = ctypes.c_int, sla.lib().mxfp4_gemm_fwd.argtypes
    xq, wq, bias = sla.mxfp4_quantize(_bf16(M, (M, K))), sla.mxfp4_quantize(_bf16(N, (N, K), K ** -0.5)), _bf16(K, N)
    got = [sla.mxfp4_gemm_fwd(xq, wq, M, N, K, bias=bias) for _ in range(3)]
    want = torch.empty_like(got[0])
    assert full(xq.data_ptr(), xq.numel(), wq.data_ptr(), wq.numel(), bias.data_ptr(), want.data_ptr(), M, N, K,
                torch.cuda.current_stream().cuda_stream) == 0
    assert all(torch.equal(y, want) for y in got)
