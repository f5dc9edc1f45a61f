"""Attention to a sequence of another length on the GPU against the float64 oracle.

Tolerances, from the roundings (a rounding to bf16 is off by at most u = 2^-8 of the value).  Forward: each weight is rounded once,
the quotient divides by the sum of the rounded ones, and the result is rounded once: |error| <= 2 u sum p |v| + u |out|, and of
that sum p |v| bounds |out| (and fp32's share, with scores of up to 40: 40 * 2^-22 of sum p |v|): 3.1 u sum p |v| in all.
lse: fp32 on scores of size s: 2^-20 (1 + |s|).
Gradients: P and dS are rounded once each, delta comes from the rounded out (off by u sum |dout| |out| + 2.1 u sum |dout| (sum p |v|)
at most), the result is rounded once.  With the sizes' sums as the oracle's helper below gives them, a bound of u times four of them."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2512_16093_amd import binding as sla

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


def _np(t):
    return t.detach().double().cpu().numpy()


def _bf16(r, shape, amp=1.0):
    return torch.from_numpy((amp * r.standard_normal(shape)).astype(np.float32)).bfloat16()


def _order(x, kind):
    """x [B, H, N, d] in one of the memory orders the library takes, on the GPU."""
    if kind == "contiguous":
        return x.cuda()
    if kind == "token":
        return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
    wide = torch.full((x.shape[0], x.shape[2], 2, x.shape[1], x.shape[3]), 7.0, dtype=torch.bfloat16, device="cuda")   # one of a packed pair
    wide[:, :, 1] = x.permute(0, 2, 1, 3).cuda()
    return wide[:, :, 1].permute(0, 2, 1, 3)


def _bounds(q, k, v, dout, out, lens, scale):
    """Per element: sum p |v|; and of the gradients' terms that are rounded, with delta's own error in them."""
    B, H, Nq, d = q.shape
    G, Nk = k.shape[1], k.shape[2]
    pv, bq, bk, bv = np.zeros(q.shape), np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape)
    for b in range(B):
        n = Nk if lens is None else min(max(int(lens[b]), 0), Nk)
        for h in range(H if n else 0):
            g = h // (H // G)
            s = q[b, h] @ k[b, g, :n].T * scale
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            pv[b, h] = p @ np.abs(v[b, g, :n])
            dp = dout[b, h] @ v[b, g, :n].T
            delta = (p * dp).sum(1, keepdims=True)
            wrong = (np.abs(dout[b, h]) * (np.abs(out[b, h]) + 2.1 * pv[b, h])).sum(1, keepdims=True)
            ds = p * (np.abs(dp - delta) + wrong) * scale
            bq[b, h] = ds @ np.abs(k[b, g, :n])
            bk[b, g, :n] += ds.T @ np.abs(q[b, h])
            bv[b, g, :n] += p.T @ np.abs(dout[b, h])
    return pv, bq, bk, bv


CASES = [  # B, H, Hkv, Nq, Nk, lens, memory order
    (1, 1, 1, 1, 1, None, "contiguous"),
    (1, 2, 1, 1, 7, None, "token"),
    (2, 2, 2, 33, 31, (31, 0), "token"),               # a sample without keys
    (3, 2, 2, 5, 64, (1, 33, 64), "packed"),
    (1, 3, 3, 64, 65, None, "contiguous"),
    (1, 2, 2, 129, 128, None, "token"),
    (2, 4, 2, 100, 77, (77, 20), "packed"),
    (1, 2, 2, 257, 512, (500,), "token"),
    (2, 12, 12, 300, 226, (226, 9), "token"),
    (1, 40, 10, 1, 1500, None, "token"),               # one token against a long memory, heads shared: split and joined
    (1, 8, 1, 3, 4097, (4000,), "contiguous"),
    (2, 5, 1, 13, 700, (0, 650), "packed"),
    (1, 6, 2, 40, 333, None, "token"),                 # wavefronts whose rows lie in two heads
    (1, 1, 1, 200, 8192, (5000,), "contiguous"),       # split, and pieces behind the last key
    (1, 1, 1, 5000, 40, None, "contiguous"),           # dk, dv split over the queries
    (2, 4, 4, 1030, 100, (100, 3), "token"),
    (1, 7, 7, 31, 1, None, "token"),
]


def _make(B, H, Hkv, Nq, Nk, lens, order, seed=0):
    r = np.random.default_rng([B, H, Hkv, Nq, Nk, seed])
    q, k, v = _bf16(r, (B, H, Nq, 128), 1.5), _bf16(r, (B, Hkv, Nk, 128), 1.5), _bf16(r, (B, Hkv, Nk, 128))
    dout = _bf16(r, q.shape, 0.01)
    dl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    return q, k, v, dout, dl


def _padded_with(x, lens, value):
    """x with `value` in every row behind a sample's length."""
    x = x.clone()
    for b, n in enumerate(lens or ()):
        x[b, :, max(n, 0):] = value
    return x


@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,lens,order", CASES)
def test_forward_and_backward(B, H, Hkv, Nq, Nk, lens, order):
    q, k, v, dout, dl = _make(B, H, Hkv, Nq, Nk, lens, order)
    scale = 128 ** -0.5
    args = [_np(t) for t in (q, k, v, dout)]
    want, want_lse = bo.xattn_fwd(*args[:3], lens)
    wants = bo.xattn_bwd(*args, lens)
    # what lies behind the last key does not matter: NaN in the values, infinities in the keys
    g = [_order(t, order) for t in (q, _padded_with(k, lens, float("inf")), _padded_with(v, lens, float("nan")), dout)]
    out, lse = sla.xattn_fwd(*g[:3], k_lens=dl, want_lse=True)
    plain, none = sla.xattn_fwd(*g[:3], k_lens=dl, out=_order(torch.zeros(q.shape, dtype=torch.bfloat16), order))
    assert none is None and torch.equal(plain, out)
    pv, bq, bk, bv = _bounds(*args, want, lens, scale)
    assert (np.abs(_np(out) - want) <= 3.1 * U * pv).all(), float(np.abs(_np(out) - want).max())
    got_lse = _np(lse)
    empty = np.isinf(want_lse)
    assert (got_lse[empty] == -np.inf).all()
    assert (np.abs(got_lse[~empty] - want_lse[~empty]) <= 2.0 ** -20 * (1 + 40.0)).all()
    grads = [_order(torch.full(t.shape, 3.0, dtype=torch.bfloat16), order) for t in (q, k, v)]
    got = sla.xattn_bwd(*g[:3], out, g[3], lse, k_lens=dl, grads=grads)
    again = sla.xattn_bwd(*g[:3], out, g[3], lse, k_lens=dl)
    for name, x, y, w, bound in zip(("dq", "dk", "dv"), got, again, wants, (bq, bk, bv)):
        err = np.abs(_np(x) - w)
        assert (err <= 4 * U * bound + 1e-30).all(), (name, float((err / (bound + 1e-30)).max()))
        assert torch.equal(x, y), name
    for b, n in enumerate(lens or ()):                   # keys that are not there have no gradient
        assert (got[1][b, :, n:] == 0).all() and (got[2][b, :, n:] == 0).all()


@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_another_scale_and_large_scores(scale):
    r = np.random.default_rng(3)
    q, k, v, dout = (_bf16(r, (1, 2, n, 128), a) for n, a in ((70, 3.0), (150, 3.0), (150, 1.0), (70, 0.01)))
    args = [_np(t) for t in (q, k, v, dout)]
    want, want_lse = bo.xattn_fwd(*args[:3], None, scale)
    wants = bo.xattn_bwd(*args, None, scale)
    g = [t.cuda() for t in (q, k, v, dout)]
    out, lse = sla.xattn_fwd(*g[:3], scale=scale, want_lse=True)
    pv, bq, bk, bv = _bounds(*args, want, None, scale)
    top = np.abs(want_lse).max()                         # scores of several hundred: fp32 is off by that much of 2^-22 in the exponent
    more = 1 + top * 2.0 ** -21 / U
    assert (np.abs(_np(out) - want) <= 3.1 * U * more * pv).all()
    assert (np.abs(_np(lse) - want_lse) <= 2.0 ** -20 * (1 + top)).all()
    for x, w, bound in zip(sla.xattn_bwd(*g[:3], out, g[3], lse, scale=scale), wants, (bq, bk, bv)):
        assert (np.abs(_np(x) - w) <= 4 * U * more * bound + 1e-30).all()


def test_lengths_out_of_range_are_clamped():
    q, k, v, dout, _ = _make(3, 2, 2, 20, 50, None, "token", 1)
    g = [t.cuda() for t in (q, k, v, dout)]
    results = []
    for lens in ((-5, 50, 7), (0, 1000, 7)):
        dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
        out, lse = sla.xattn_fwd(*g[:3], k_lens=dl, want_lse=True)
        results.append((out, lse, *sla.xattn_bwd(*g[:3], out, g[3], lse, k_lens=dl)))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert (results[0][0][0] == 0).all() and (results[0][2][0] == 0).all()


def test_broadcast_inputs_and_rows_around_an_output():
    """Strides of zero (one head, one sample for all), outputs inside larger tensors that keep the rest."""
    r = np.random.default_rng(4)
    q = _bf16(r, (1, 1, 45, 128)).cuda().expand(2, 3, 45, 128)
    k, v = (_bf16(r, (1, 1, 90, 128)).cuda().expand(2, 3, 90, 128) for _ in range(2))
    around = torch.full((2, 3, 60, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    out, lse = sla.xattn_fwd(q, k, v, out=around[:, :, 7:52], want_lse=True)
    want, _ = sla.xattn_fwd(q.contiguous(), k.contiguous(), v.contiguous())
    assert torch.equal(out, want) and (around[:, :, :7] == 5).all() and (around[:, :, 52:] == 5).all()
    dk = torch.full((2, 3, 100, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    dv = dk.clone()
    a = sla.xattn_bwd(q, k, v, out, q, lse, grads=(torch.empty_like(want), dk[:, :, 3:93], dv[:, :, 3:93]))
    b = sla.xattn_bwd(q.contiguous(), k.contiguous(), v.contiguous(), want, q.contiguous(), lse)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    for t in (dk, dv):
        assert (t[:, :, :3] == 5).all() and (t[:, :, 93:] == 5).all()


def test_another_stream_and_a_captured_graph():
    q, k, v, dout, _ = _make(2, 4, 2, 70, 1200, None, "token", 2)
    lens = torch.tensor((1200, 100), dtype=torch.int32, device="cuda")
    g = [_order(t, "token") for t in (q, k, v, dout)]

    def calls():
        out, lse = sla.xattn_fwd(*g[:3], k_lens=lens, want_lse=True)
        return [out, lse, *sla.xattn_bwd(*g[:3], out, g[3], lse, k_lens=lens)]

    eager = calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for seed in range(3):
        r = np.random.default_rng([11, seed])
        for t in g:
            t.copy_(_bf16(r, t.shape))
        lens.copy_(torch.tensor((1000 - 300 * seed, 1200 * (seed % 2)), dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in held]
        assert all(torch.equal(a, b) for a, b in zip(replayed, calls())), seed
