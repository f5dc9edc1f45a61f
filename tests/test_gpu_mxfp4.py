"""Microscaled 4-bit floating point on the GPU: codes and exponents bit for bit against the float64 oracle, the product
against one in 64 bits of the values that the codes stand for.

Tolerance of the product.  Products of two values are exact (at most 4 significant bits, scaled by powers of two).  They are added
up in fp32: in every step of 64 features at most 7 additions deep (64 terms in pairs, then the accumulator), each off by at most 2^-23 of
the sizes added so far even where it cuts instead of rounding; joining the parts of a contraction that was split adds up to 8 more, the bias one.  So
a sum is off by at most (7 ceil(K / 64) + 9) 2^-23 of the sum of its terms' sizes, and its rounding to bf16 by 2^-8 of the result."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mo
from paper_2512_16093_amd import binding as sla

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def _np(t):
    return t.detach().double().cpu().numpy()


def _bf16(r, shape, amp=1.0):
    return torch.from_numpy((amp * r.standard_normal(shape)).astype(np.float32)).bfloat16()


def _held(q, R, K):
    codes, exps = sla.mxfp4_unpack(q, R, K)
    return mo.codes_of(codes.cpu().numpy()), exps.cpu().numpy()


def test_every_bf16_number_under_every_fit_of_its_block():
    """All finite bf16 magnitudes of both signs, in blocks of neighbours: the largest of a block has any mantissa, the others lie
    near it (all 15 codes' borders are met); and each number beside one four times as large."""
    bits = np.arange(0, 0x7F80, dtype=np.uint16)
    r = np.random.default_rng(1)
    rows = []
    for shift in range(4):
        n = np.roll(bits, 7 * shift)
        rows.append(n.reshape(-1, 32))
    wide = np.stack([np.minimum(bits[i::64][:510], 0x7F7F) for i in range(64)])          # blocks that span many binades
    rows.append(wide.reshape(-1, 30)[:, :30].repeat(2, 1)[:, :32])
    four = np.stack((bits, np.where(bits < 0x7E80, bits + 0x100, 0x7F7F)), 1).reshape(-1, 2).astype(np.uint16)
    rows.append(np.tile(four, (1, 16)))
    x = np.concatenate(rows).astype(np.uint16)
    x ^= (r.integers(0, 2, x.shape) << 15).astype(np.uint16)
    R = x.shape[0]
    t = torch.from_numpy(x.view(np.int16).copy()).view(torch.bfloat16)
    codes, exps = _held(sla.mxfp4_quantize(t.cuda()), R, 32)
    want, want_exps = mo.quantize(_np(t))
    assert (exps == want_exps).all()
    bad = codes != want
    assert not bad.any(), (bad.sum(), x[bad.any(1)][:2], codes[bad][:8], want[bad][:8])


SHAPES = [(1, 8), (1, 32), (3, 40), (31, 256), (32, 264), (33, 248), (7, 1000), (65, 512), (130, 1536), (9, 8192), (2, 65536), (1000, 104)]


@pytest.mark.parametrize("R,K", SHAPES)
def test_quantise_and_back(R, K):
    r = np.random.default_rng([R, K])
    x = (_bf16(r, (R, K)).float() * torch.from_numpy(10.0 ** r.integers(-20, 20, (R, 1))).float()).bfloat16()
    x[:, ::29] *= 12
    x[R // 2, : K // 2] = 0
    nbytes = sla.mxfp4_bytes(R, K)
    around = torch.full((nbytes + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    q = sla.mxfp4_quantize(x.cuda(), around[:nbytes])
    assert (around[nbytes:] == 0xA5).all()
    codes, exps = _held(q, R, K)
    want, want_exps = mo.quantize(_np(x))
    assert (exps == want_exps).all() and (codes == want).all()
    out = torch.full((R + 1, K), 7.0, dtype=torch.bfloat16, device="cuda")
    back = sla.mxfp4_dequantize(q, R, K, out[:R])
    assert (_np(back) == mo.dequantize(want, want_exps)).all() and (out[R] == 7).all()
    # plain rows in and out again
    c, e = sla.mxfp4_unpack(q, R, K)
    again = sla.mxfp4_pack(c, e)
    c2, e2 = sla.mxfp4_unpack(again, R, K)
    assert torch.equal(c, c2) and torch.equal(e, e2) and torch.equal(sla.mxfp4_dequantize(again, R, K), back)


def test_blocks_that_hold_no_number_and_the_ends_of_the_exponents():
    r = np.random.default_rng(3)
    x = _bf16(r, (6, 104))
    x[1, 40], x[2, 103], x[3, 0], x[4, 64] = float("nan"), float("inf"), float("-inf"), 3.3e38
    x[5, 0:32], x[5, 32:64] = 1e-38, 0.0
    codes, exps = _held(sla.mxfp4_quantize(x.cuda()), 6, 104)
    want, want_exps = mo.quantize(_np(x))
    assert (exps == want_exps).all() and (codes == want).all() and (exps == 255).sum() == 3
    back = _np(sla.mxfp4_dequantize(sla.mxfp4_quantize(x.cuda()), 6, 104))
    assert np.array_equal(back, mo.dequantize(want, want_exps), equal_nan=True)
    # every exponent and code, as another program may hand them over; what is beyond bf16 is an infinity
    codes = np.tile(np.arange(16, dtype=np.uint8), (256, 2))
    exps = np.arange(256, dtype=np.uint8)[:, None]
    q = sla.mxfp4_pack(torch.from_numpy(mo.plain(codes)).cuda(), torch.from_numpy(exps).cuda())
    want = mo.dequantize(codes, exps)
    want = np.where(np.abs(want) > 3.39e38, np.sign(want) * np.inf, want)
    assert np.array_equal(_np(sla.mxfp4_dequantize(q, 256, 32)), want, equal_nan=True)


def _product(xq, wq, M, N, K, bias):
    """(the layer in 64 bits of what the objects hold, the sizes of its terms)"""
    a, b = (mo.dequantize(*_held(q, R, K)) for q, R in ((xq, M), (wq, N)))
    y, size = a @ b.T, np.abs(a) @ np.abs(b).T
    return (y, size) if bias is None else (y + _np(bias), size + np.abs(_np(bias)))


def _check(y, want, size, K):
    bad = ~(np.abs(_np(y) - want) <= HALF * np.abs(want) + (7 * -(-K // 64) + 9) * 2.0 ** -23 * size + 1e-37)
    assert not bad.any(), "%d of %d off, worst %.3e" % (bad.sum(), bad.size, np.abs(_np(y) - want).max())


GEMM = [  # M, N, K
    (1, 8, 8), (1, 32, 32), (1, 1536, 256), (1, 5120, 5120), (2, 40, 2000), (5, 264, 520), (16, 1000, 1536), (31, 96, 64), (32, 256, 1024),
    (33, 136, 264), (64, 512, 8960), (65, 5120, 1536), (127, 72, 776), (128, 128, 512), (130, 1304, 4096), (200, 2048, 256), (256, 256, 2048),
    (257, 264, 1000), (300, 8, 13824), (512, 1536, 5120), (700, 2056, 1544), (1025, 768, 640), (1500, 1536, 1280), (2100, 2600, 512),
    (4099, 520, 72), (3, 8960, 16384), (40, 15360, 136),
]


LARGE = [  # every kernel of the larger calls: square tiles (4 and 3 stages), wide, walked; one step, two and more; few and many token
    # tiles; edges of tokens and outputs
    (1000, 1032, 200), (1000, 1032, 400), (1000, 1032, 520), (1100, 1304, 776), (1100, 1304, 1800),
    (2100, 2184, 136), (2100, 2184, 264), (3000, 1800, 520), (2300, 2056, 1536),
    (5000, 4104, 200), (5000, 4104, 400), (33000, 520, 520), (33000, 520, 776),
    (8200, 8200, 1000), (66000, 776, 1280), (8193, 8192, 1288), (65600, 1032, 1024),
]


@pytest.mark.parametrize("M,N,K", GEMM + LARGE)
def test_linear(M, N, K):
    r = np.random.default_rng([M, N, K])
    x, w, bias = _bf16(r, (M, K), 2.0), _bf16(r, (N, K), K ** -0.5), _bf16(r, N, 0.5).cuda()
    x[:, ::31] *= 15
    x, w = x.cuda(), w.cuda()
    xq, wq = sla.mxfp4_quantize(x), sla.mxfp4_quantize(w)
    out = torch.full((M + 1, N), 7.0, dtype=torch.bfloat16, device="cuda")
    y = sla.mxfp4_linear_fwd(x, wq, N, bias=bias, out=out[:M])
    assert (out[M] == 7).all()
    _check(y, *_product(xq, wq, M, N, K, bias), K)
    assert torch.equal(y, sla.mxfp4_linear_fwd(x, wq, N, bias=bias))
    g = sla.mxfp4_gemm_fwd(xq, wq, M, N, K)
    _check(g, *_product(xq, wq, M, N, K, None), K)
    assert torch.equal(g, sla.mxfp4_gemm_fwd(xq, wq, M, N, K))
    _check(sla.mxfp4_gemm_fwd(xq, wq, M, N, K, bias=bias), *_product(xq, wq, M, N, K, bias), K)


@pytest.mark.parametrize("M,N,K", [(1, 512, 768), (3, 40, 264), (70, 264, 1032), (600, 1040, 512), (4100, 2056, 776)])
def test_rows_and_outputs_that_are_no_numbers_stay_by_themselves(M, N, K):
    """A NaN among the activations makes its row NaN, one in the weight its output; the objects' rows behind the last hold anything."""
    r = np.random.default_rng([M, N, K])
    x, w = _bf16(r, (M, K)).cuda(), _bf16(r, (N, K), K ** -0.5).cuda()
    clean = sla.mxfp4_linear_fwd(x, sla.mxfp4_quantize(w), N)
    poisoned = lambda R: torch.full((sla.mxfp4_bytes(R, K),), 0xFF, dtype=torch.uint8, device="cuda")
    x2, w2 = x.clone(), w.clone()
    x2[M // 2, K - 1] = float("nan")
    w2[N - 1, 0] = float("inf")
    y = sla.mxfp4_linear_fwd(x2, sla.mxfp4_quantize(w2, poisoned(N)), N, workspace=poisoned(M))
    rows, cols = [i for i in range(M) if i != M // 2], list(range(N - 1))
    assert torch.isnan(y[M // 2]).all() and torch.isnan(y[:, N - 1]).all()
    assert torch.equal(y[rows][:, cols], clean[rows][:, cols])
    g = sla.mxfp4_gemm_fwd(sla.mxfp4_quantize(x2, poisoned(M)), sla.mxfp4_quantize(w2, poisoned(N)), M, N, K)
    assert torch.isnan(g[M // 2]).all() and torch.isfinite(g[rows][:, cols]).all()


def test_exponents_far_apart_in_a_row_and_of_another_program():
    """Blocks of very different size along the contraction, exponents from one end to the other in activations and weights."""
    M, N, K = 40, 72, 512
    r = np.random.default_rng(12)
    codes = [r.integers(0, 16, (R, K)).astype(np.uint8) for R in (M, N)]
    e = r.integers(60, 190, (1, K // 32))
    exps = [np.broadcast_to(e, (M, K // 32)).astype(np.uint8), np.broadcast_to(254 - e, (N, K // 32)).astype(np.uint8)]
    q = [sla.mxfp4_pack(torch.from_numpy(mo.plain(c)).cuda(), torch.from_numpy(np.ascontiguousarray(s)).cuda()) for c, s in zip(codes, exps)]
    y = sla.mxfp4_gemm_fwd(q[0], q[1], M, N, K)
    _check(y, *_product(q[0], q[1], M, N, K, None), K)


LAYER = [(1, 1, 8), (1, 1, 5120), (2, 8, 1536), (1, 5, 1000), (3, 11, 2056), (1, 70, 264), (2, 40, 8200), (1, 3, 16384), (1, 33, 6144 + 8), (4, 301, 1536)]


@pytest.mark.parametrize("S,rows,K", LAYER)
@pytest.mark.parametrize("full", [False, True])
def test_norm_in_front_of_a_layer(S, rows, K, full):
    r = np.random.default_rng([S, rows, K])
    M, N = S * rows, 264
    x, v = _bf16(r, (M, K), 2.0).cuda(), {}
    if full:
        six = torch.from_numpy((0.4 * r.standard_normal((S, 6, K))).astype(np.float32)).cuda()
        v = dict(res=_bf16(r, (M, K)).cuda(), gate=six[:, 5], scale=six[:, 1], shift=six[:, 0])
    nw, nb = ((1 + 0.2 * _bf16(r, K)).bfloat16().cuda(), _bf16(r, K).cuda()) if full else (None, None)
    y, h = sla.norm_layer_fwd(x, nw, nb, **v)
    q, h2 = sla.mxfp4_norm_quantize(x, nw, nb, **v)
    assert torch.equal(h, h2)
    a, b = sla.mxfp4_unpack(q, M, K), sla.mxfp4_unpack(sla.mxfp4_quantize(y), M, K)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    wq, bias = sla.mxfp4_quantize(_bf16(r, (N, K), K ** -0.5).cuda()), _bf16(r, N).cuda()
    out, h3 = sla.mxfp4_norm_linear_fwd(x, wq, N, nw, nb, **v, bias=bias)
    assert torch.equal(h, h3) and torch.equal(out, sla.mxfp4_gemm_fwd(q, wq, M, N, K, bias=bias))
    _check(out, *_product(q, wq, M, N, K, bias), K)


def test_a_block_of_these_operators_on_streams_and_in_graphs():
    """Norm into a layer, its result through the gate into the stream and into the next layer, as a DiT block runs them; on a side
    stream, and recorded into two graphs that share no workspace but run in turn, replayed on fresh inputs."""
    S, rows, K, F = 2, 70, 1536, 4104
    r = np.random.default_rng(9)
    M = S * rows
    x = _bf16(r, (M, K)).cuda()
    six = torch.from_numpy((0.4 * r.standard_normal((S, 6, K))).astype(np.float32)).cuda()
    w1, w2, wp = (sla.mxfp4_quantize(_bf16(r, s, 0.03).cuda()) for s in ((F, K), (K, F), (K, K)))
    dy = _bf16(r, (M, K)).cuda()

    def calls():
        n, _ = sla.mxfp4_norm_linear_fwd(x, wp, K, scale=six[:, 1], shift=six[:, 0])
        up, h = sla.mxfp4_norm_linear_fwd(x, w1, F, res=n, gate=six[:, 2], scale=six[:, 4], shift=six[:, 3])
        down = sla.mxfp4_linear_fwd(up, w2, K)
        y, h2 = sla.norm_layer_fwd(h, res=down, gate=six[:, 5])
        return [n, up, h, down, y, h2, *[t for t in sla.norm_layer_bwd(dy, h2, res=down, gate=six[:, 5]) if t is not None]]
    eager = [t.clone() for t in calls()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, calls()))
    for seed in range(3):
        r = np.random.default_rng([10, seed])
        x.copy_(_bf16(r, (M, K)))
        six.copy_(torch.from_numpy((0.4 * r.standard_normal((S, 6, K))).astype(np.float32)))
        for g, held in graphs + graphs[:1]:
            g.replay()
            torch.cuda.synchronize()
            replayed = [t.clone() for t in held]
            assert all(torch.equal(a, b) for a, b in zip(replayed, calls())), seed


@pytest.mark.parametrize("M,N,K", [(512, 13824, 2312), (1023, 5128, 2056), (300, 13832, 4096), (1800, 5120, 2304), (700, 5120, 2560), (1024, 15360, 2312), (2040, 13824, 2056), (5000, 5128, 2056)])
def test_large_tiles_that_are_few(M, N, K):
    """Contractions of more than 2048 features in one and two rounds of wide or walked tiles, and calls that keep the square ones."""
    test_linear(M, N, K)


def test_calls_at_once_and_graphs_that_share_a_workspace():
    """Two chains on two streams at the same time, each with workspaces of its own; two graphs captured over one workspace, replayed in
    turn on one stream."""
    K, N = 1536, 2056
    r = np.random.default_rng(21)
    wq = sla.mxfp4_quantize(_bf16(r, (N, K), 0.03).cuda())
    xs = [_bf16(r, (M, K)).cuda() for M in (3000, 700)]
    res = [_bf16(r, x.shape).cuda() for x in xs]
    call = lambda i, ws=None: [*sla.mxfp4_norm_linear_fwd(xs[i], wq, N, res=res[i], workspace=ws), *sla.norm_layer_bwd(xs[i], res[i], dh=xs[i])[:1]]
    alone = [[t.clone() for t in call(i)] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    at_once = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                at_once[i].append(call(i))
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for got in at_once[i] for a, b in zip(got, alone[i]))
    shared = torch.full((sla.mxfp4_bytes(3000, K),), 0xFF, dtype=torch.uint8, device="cuda")
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, call(i, shared)))
    for i in (0, 1, 1, 0, 1, 0):
        for t in graphs[i][1]:
            t.zero_()
        shared.fill_(0xFF)
        graphs[i][0].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(graphs[i][1], alone[i])), i
