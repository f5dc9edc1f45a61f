"""Attention to a sequence of another length at the ends of its range, in every way its work is dealt out: numbers that are none, the
largest scores, samples of enough units to be dealt one after the other."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2512_16093_amd import binding as sla
from test_gpu_xattn import U, _bounds, _make, _order, _padded_with

pytestmark = pytest.mark.gpu


def _bf16(r, shape, amp=1.0):
    return torch.from_numpy((amp * r.standard_normal(shape)).astype(np.float32)).bfloat16()


def _pieces(B, H, Hkv, Nq, Nk):
    """In how many pieces the forward walk is split: what the workspace holds (fp32 rows of 128 + 4)."""
    return max(1, sla.xattn_workspace_bytes(B, H, Hkv, Nq, Nk, 128) // (B * H * Nq * 132 * 4))


WALKS = [  # B, H, Hkv, Nq, Nk, lens, fewest and most pieces: one walk; a few, joined side by side; many, joined in turn
    (2, 2, 2, 130, 100, (100, 70), 1, 1),
    (1, 24, 24, 300, 1500, (1490,), 2, 8),
    (2, 8, 2, 3, 2500, (2500, 2100), 9, 1024),
]


@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,lens,least,most", WALKS)
def test_nan_stays_nan(B, H, Hkv, Nq, Nk, lens, least, most):
    """A NaN in a query, or in a key that counts, is NaN in the rows that meet it, their log-sum-exp included (-infinity would
    say that they have no keys); one in a value is NaN in its channel.  Every other number is what it was."""
    assert least <= _pieces(B, H, Hkv, Nq, Nk) <= most
    r = np.random.default_rng([B, H, Nq])
    q, k, v = (_bf16(r, s).cuda() for s in ((B, H, Nq, 128), (B, Hkv, Nk, 128), (B, Hkv, Nk, 128)))
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = sla.xattn_fwd(q, k, v, k_lens=dl, want_lse=True)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()

    def same_but(got, want, where):
        assert torch.isnan(got[where]).all()
        assert torch.equal(got[~where], want[~where])

    nan, group = float("nan"), H // Hkv
    for row in {0, Nq - 1}:
        bad = q.clone()
        bad[0, 1, row, 5] = nan
        where = torch.zeros_like(lse, dtype=torch.bool)
        where[0, 1, row] = True
        got, got_lse = sla.xattn_fwd(bad, k, v, k_lens=dl, want_lse=True)
        same_but(got_lse, lse, where)
        same_but(got, out, where[..., None].expand_as(out))
        assert torch.equal(sla.xattn_fwd(bad, k, v, k_lens=dl)[0].isnan(), got.isnan())
    for key in (0, lens[0] - 1):
        bad = k.clone()
        bad[0, Hkv - 1, key, 100] = nan
        where = torch.zeros_like(lse, dtype=torch.bool)
        where[0, H - group:] = True
        got, got_lse = sla.xattn_fwd(q, bad, v, k_lens=dl, want_lse=True)
        same_but(got_lse, lse, where)
        same_but(got, out, where[..., None].expand_as(out))
        bad = v.clone()
        bad[0, Hkv - 1, key, 100] = nan
        where = torch.zeros_like(out, dtype=torch.bool)
        where[0, H - group:, :, 100] = True
        got, got_lse = sla.xattn_fwd(q, k, bad, k_lens=dl, want_lse=True)
        assert torch.equal(got_lse, lse)
        same_but(got, out, where)


def _np(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,lens,least,most", WALKS)
def test_the_largest_scores(B, H, Hkv, Nq, Nk, lens, least, most):
    """Scores of just below 2^24 either way, which fp32 holds exactly here (whole numbers), a few units apart where they count.
    Tolerances: 3.1 roundings to bf16 of sum p |v| (test_gpu_xattn.py), and of the exponents, up to 7 log2(e) apart, what fp32 adds to
    them (far below one); lse: the rounding of a number of its size, its two factors and its sum's, 2^-22 in all."""
    r = np.random.default_rng([B, H, Nk])
    q, k = torch.zeros((B, H, Nq, 128)), torch.zeros((B, Hkv, Nk, 128))
    q[..., 3] = torch.from_numpy(r.choice((-1.0, 1.0), (B, H, Nq))) * 2.0 ** 14        # times 1020: 2^24 - 2^16
    q[..., 77] = 1.0
    k[..., 3] = torch.from_numpy(r.choice((1020.0, 1020.0, 1016.0, -1020.0), (B, Hkv, Nk)))
    k[0, 0, :, 3] = 1020.0                                                             # (rows whose scores are all the lowest)
    k[..., 77] = torch.from_numpy(r.integers(0, 8, (B, Hkv, Nk)).astype(np.float64))
    q, k, v = q.bfloat16(), k.bfloat16(), _bf16(r, (B, Hkv, Nk, 128))
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = sla.xattn_fwd(q.cuda(), k.cuda(), v.cuda(), k_lens=dl, scale=1.0, want_lse=True)
    args = [_np(t) for t in (q, k, v)]
    want, want_lse = bo.xattn_fwd(*args, lens, 1.0)
    size = bo.xattn_fwd(args[0], args[1], np.abs(args[2]), lens, 1.0)[0]
    assert (np.abs(_np(out) - want) <= 3.1 * 2.0 ** -8 * size).all()
    assert (np.abs(_np(lse) - want_lse) <= 2.0 ** -22 * np.abs(want_lse)).all()


@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,lens,order", [   # units per sample: forward, dq, dk and dv (on 256 compute units)
    (3, 5, 5, 1700, 100, (100, 0, 57), "token"),         # 70, 70 (no eighths), 45
    (3, 2, 2, 100, 4800, (4800, 0, 2500), "contiguous"), # 50, 50, 76
    (2, 11, 11, 300, 1500, (1500, 700), "packed"),       # 99, 165 (pieces), 132
    (2, 13, 13, 40, 300, (9, 300), "token"),             # 65, 65 (pieces behind a sample's last key), 39
    (3, 6, 3, 3000, 70, (70, 0, 33), "token"),           # 141, 141, 72 (pieces; heads shared)
    (2, 7, 7, 1300, 400, None, "packed"),                # 77, 77, 112
])
def test_samples_of_many_units(B, H, Hkv, Nq, Nk, lens, order):
    """A sample of 64 units or more is spread over the whole chip by itself, the next one after it: every row of every sample is
    written, and right.  (Tolerances: test_gpu_xattn.py.)"""
    q, k, v, dout, dl = _make(B, H, Hkv, Nq, Nk, lens, order)
    args = [_np(t) for t in (q, k, v, dout)]
    want, want_lse = bo.xattn_fwd(*args[:3], lens)
    wants = bo.xattn_bwd(*args, lens)
    pv, bq, bk, bv = _bounds(*args, want, lens, 128 ** -0.5)
    nan = float("nan")
    g = [_order(t, order) for t in (q, _padded_with(k, lens, nan), _padded_with(v, lens, nan), dout)]
    fresh = lambda t: _order(torch.full(t.shape, nan, dtype=torch.bfloat16), order)
    out, lse = sla.xattn_fwd(*g[:3], k_lens=dl, want_lse=True, out=fresh(q))
    assert (np.abs(_np(out) - want) <= 3.1 * U * pv).all()
    empty = np.isinf(want_lse)
    assert (_np(lse)[empty] == -np.inf).all()
    assert (np.abs(_np(lse)[~empty] - want_lse[~empty]) <= 2.0 ** -20 * (1 + 40.0)).all()
    got = sla.xattn_bwd(*g[:3], out, g[3], lse, k_lens=dl, grads=[fresh(t) for t in (q, k, v)])
    for name, x, w, bound in zip(("dq", "dk", "dv"), got, wants, (bq, bk, bv)):
        assert (np.abs(_np(x) - w) <= 4 * U * bound + 1e-30).all(), name
