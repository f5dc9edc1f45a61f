"""Attention to a sequence of another length: numbers that are none, in every way the walk over the keys is dealt out."""
import numpy as np
import pytest
import torch

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
