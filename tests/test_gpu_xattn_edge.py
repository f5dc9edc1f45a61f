"""Attention to a sequence of another length at the ends of its range, in every way the walk over the keys is dealt out: numbers that
are none, the largest scores."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2512_16093_amd import binding as sla

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
