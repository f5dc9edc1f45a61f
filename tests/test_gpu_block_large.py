"""The block's operators at the largest model's sizes, and where offsets pass 32 bits: samples against float64."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2512_16093_amd import binding as sla

pytestmark = pytest.mark.gpu
U, F32 = 2.0 ** -8, 2.0 ** -19       # half a step of bf16; what fp32 adds to the terms (test_gpu_rope_norm.py)


def _np(t):
    return t.detach().double().cpu().numpy()


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def _normal(shape, seed, amp=1.0):
    """bf16 normal values, formed a slab at a time."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    for part in x.view(-1).split(1 << 27):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(amp))
    return x


@pytest.mark.parametrize("N,H", [(75600, 40), (280000, 32)])       # (a packed projection of 2.3 and of 6.9 GB)
def test_rope_on_a_large_packed_projection(N, H):
    x = _normal((1, N, 3, H, 128), N, 1.7)
    q, k = (x[:, :, i].permute(0, 2, 1, 3) for i in (0, 2))
    n = torch.arange(N, device="cuda")
    pos = torch.stack((n // 3600, n // 80 % 45, n % 80), 1).int().contiguous()
    w = [(1 + 0.2 * _normal((H * 128,), s)).bfloat16() for s in (1, 2)]
    got = sla.rope_qk_fwd(q, k, pos, sla.rope_make_plan(), w[0], w[1], "token")
    back = sla.rope_qk_bwd(got[0], got[1], pos, sla.rope_make_plan(), q, k, w[0], w[1], "token")
    some = torch.tensor([0, 1, 3, 4, N // 2, N - 2, N - 1], device="cuda")
    ang = bo.angles(pos[some].cpu().numpy()[None], (22, 21, 21), (10000.0,) * 3)
    for i, src in enumerate((q, k)):
        x64, y64 = _np(src[:, :, some]), _np(got[i][:, :, some])
        want = bo.rope_fwd(x64, ang, "interleaved", _np(w[i]), "token")
        size = np.abs(bo.rope_fwd(x64, ang * 0, "interleaved", _np(w[i]), "token"))
        scale = np.repeat(size[..., 0::2] + size[..., 1::2], 2, -1)
        assert (np.abs(y64 - want) <= U * np.abs(want) + F32 * scale).all()
        dx, _, scale = bo.rope_bwd(y64, x64, ang, "interleaved", _np(w[i]), "token")
        assert (np.abs(_np(back[i][:, :, some]) - dx) <= U * np.abs(dx) + F32 * scale).all()


def test_norm_of_more_than_4_gb():
    M, K = 600_000, 4096
    x, res = _normal((M, K), 1, 2.0), _normal((M, K), 2, 0.5)
    w = (1 + 0.2 * _normal((K,), 3)).bfloat16()
    y, h = sla.norm_rms_fwd(x, w, res)
    dx, dw = sla.norm_rms_bwd(res, h, w, dh=x)
    some = torch.tensor([0, 1, 255, M // 2, 524_288, M - 1], device="cuda")      # (row 524288 starts 4 GiB on)
    assert torch.equal(h[some], (x[some].float() + res[some].float()).bfloat16())
    want = bo.norm_fwd(_np(h[some]), _np(w), 1e-6)
    assert (np.abs(_np(y[some]) - want) <= (U + F32) * np.abs(want)).all()
    want, _, scale = bo.norm_bwd(_np(res[some]), _np(h[some]), _np(w), _np(x[some]), 1e-6)
    assert (np.abs(_np(dx[some]) - want) <= U * np.abs(want) + F32 * scale).all()
    total = torch.zeros(K, dtype=torch.float64, device="cuda")
    terms = torch.zeros_like(total)
    for r0 in range(0, M, 50_000):
        v = h[r0:r0 + 50_000].double()
        t = res[r0:r0 + 50_000].double() * v * torch.rsqrt((v * v).mean(1, keepdim=True) + 1e-6)
        total += t.sum(0)
        terms += t.abs().sum(0)
    # a team adds up some 600 rows one after the other, errors of random sign: far below 600 halves of a step of the sum of sizes
    assert ((dw.double() - total).abs() <= 600 * 2.0 ** -24 * terms).all()
    ws, h2 = sla.w8a8_norm_quantize_act(x, w, res=res)
    assert torch.equal(h2, h)
    codes, scales = sla.w8a8_debug_unpack(ws, False, M, K)
    last = slice(M // 128 * 128, M)
    n = bo.norm_fwd(_np(h[last]), _np(w), 1e-6)
    amax = np.abs(n.reshape(-1, K // 128, 128)).max((0, 2)) / 127
    assert (np.abs(_np(scales[-1]) - amax) <= F32 * amax).all()
    assert (np.abs(_np(codes[last]) - n / np.repeat(amax, 128)) <= 0.5 + 127 * 2 * F32).all()


def test_cross_attention_of_the_large_model():
    """75600 queries of 40 heads to 512 states: sampled queries against float64, forward and backward (dk, dv of two heads whole)."""
    H, Nq, Nk = 40, 75600, 512
    q, k, v = (_normal((1, n, H, 128), s, a).permute(0, 2, 1, 3) for n, s, a in ((Nq, 1, 1.5), (Nk, 2, 1.5), (Nk, 3, 1.0)))
    dout = _normal((1, Nq, H, 128), 4, 0.01).permute(0, 2, 1, 3)
    out, lse = sla.xattn_fwd(q, k, v, want_lse=True)
    dq, dk, dv = sla.xattn_bwd(q, k, v, out, dout, lse)
    some = torch.tensor([0, 31, 32, 127, 128, 40000, Nq - 81, Nq - 1], device="cuda")
    a = [_np(t) for t in (q[:, :, some], k, v, dout[:, :, some])]
    want, want_lse = bo.xattn_fwd(*a[:3])
    rel = lambda got, want: np.linalg.norm(_np(got) - want) / np.linalg.norm(want)
    # roundings of P, dS and the results: 2^-9 in the mean at most each, two on the way (delta's a third for dq and dk)
    assert rel(out[:, :, some], want) < 2 * 2 ** -9 and np.abs(_np(lse[:, :, some]) - want_lse).max() < 2 ** -20 * 41
    assert rel(dq[:, :, some], bo.xattn_bwd(*a)[0]) < 3 * 2 ** -9
    for h in (0, 39):
        q64, k64, v64, d64 = (t[0, h].double() for t in (q, k, v, dout))
        p = torch.softmax(q64 @ k64.t() * 128 ** -0.5, 1)
        dp = d64 @ v64.t()
        ds = p * (dp - (p * dp).sum(1, keepdim=True)) * 128 ** -0.5
        assert rel(dv[0, h], _np(p.t() @ d64)) < 2 * 2 ** -9 and rel(dk[0, h], _np(ds.t() @ q64)) < 3 * 2 ** -9


def test_cross_attention_to_a_memory_beyond_4_gb():
    """One token (and three of a shared head) against 17 million states: offsets pass 32 bits."""
    Nk = 17_000_000
    k, v = _normal((1, 1, Nk, 128), 1), _normal((1, 1, Nk, 128), 2)
    k[0, 0, -3:] *= 3.0                                    # the last ones count
    q = _normal((1, 2, 3, 128), 3, 2.0)
    lens = torch.tensor([Nk - 1], dtype=torch.int32, device="cuda")
    out, lse = sla.xattn_fwd(q, k, v, k_lens=lens, want_lse=True)
    m = torch.full((6, 1), -float("inf"), dtype=torch.float64, device="cuda")
    l, acc = torch.zeros_like(m), torch.zeros((6, 128), dtype=torch.float64, device="cuda")
    for k0 in range(0, Nk - 1, 1 << 20):
        k1 = min(k0 + (1 << 20), Nk - 1)
        s = q.view(6, 128).double() @ k[0, 0, k0:k1].double().t() * 128 ** -0.5
        new = torch.maximum(m, s.amax(1, keepdim=True))
        p = torch.exp(s - new)
        acc = acc * torch.exp(m - new) + p @ v[0, 0, k0:k1].double()
        l = l * torch.exp(m - new) + p.sum(1, keepdim=True)
        m = new
    want, want_lse = acc / l, (m + l.log()).view(1, 2, 3)
    # 17 million weights of a few 10^-6 each: their roundings average out, the result's (2^-9 in the mean) and sums of 17 million in fp32
    # (pieces of some 17000 keys, errors of random sign, below 17000^(1/2) 2^-24 of the sizes' sum, here 1 against a result of 2^-8) remain
    assert float((out.view(6, 128).double() - want).norm() / want.norm()) < 2 ** -7
    assert float((lse.double() - want_lse).abs().max()) < 2 ** -20 * 41


def test_cross_attention_with_far_token_strides():
    """Keys 64 MB apart: the copies' 32-bit offsets do not reach."""
    Nk, far = 45, 1 << 25
    buf = torch.zeros(Nk * far, dtype=torch.bfloat16, device="cuda")
    k, v = buf.as_strided((1, 1, Nk, 128), (0, 0, far, 1)), buf.as_strided((1, 1, Nk, 128), (0, 0, far, 1), 256)
    k.copy_(_normal((1, 1, Nk, 128), 1, 1.5))
    v.copy_(_normal((1, 1, Nk, 128), 2))
    q, dout = _normal((1, 1, 77, 128), 3, 1.5), _normal((1, 1, 77, 128), 4, 0.01)
    out, lse = sla.xattn_fwd(q, k, v, want_lse=True)
    want = sla.xattn_fwd(q, k.contiguous(), v.contiguous(), want_lse=True)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    for a, b in zip(sla.xattn_bwd(q, k, v, out, dout, lse), sla.xattn_bwd(q, k.contiguous(), v.contiguous(), out, dout, lse)):
        assert torch.equal(a, b)
    # and queries that far apart
    qf, df = buf.as_strided((1, 1, 40, 128), (0, 0, far, 1), 512), buf.as_strided((1, 1, 40, 128), (0, 0, far, 1), 768)
    qf.copy_(q[:, :, :40])
    df.copy_(dout[:, :, :40])
    a = sla.xattn_bwd(qf, k, v, out[:, :, :40].contiguous(), df, lse[:, :, :40].contiguous())
    b = sla.xattn_bwd(q[:, :, :40].contiguous(), k.contiguous(), v.contiguous(), out[:, :, :40].contiguous(), dout[:, :, :40].contiguous(),
                      lse[:, :, :40].contiguous())
    assert all(torch.equal(x, y) for x, y in zip(a, b))
