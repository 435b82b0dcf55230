"""Steps over a cache in 4 bits whose values and scores spread over many powers of two: what is added up in scaled units stays in range."""
import math

import pytest
import torch

from paper_2607_24788_b200 import glide
from tests.paged_more_util import BF16, Cache4, reference4
from tests.paged_util import check

pytestmark = pytest.mark.gpu


def grown(slots, small, factor, score, H, d):
    """One sequence whose first `small` slots have keys of 0, the others keys that score `score` (log2); values on 16 levels with a step of 1.875 behind them,
    of 1 / factor in them."""
    g = torch.Generator().manual_seed(1)
    u = (torch.randint(0, 2, (d,), generator=g) * 2 - 1).cuda()

    def rows(b, k, v):
        n = len(k)
        at = torch.arange(n, device="cuda")[:, None, None]
        a = score * math.log(2.0) / d ** 0.5
        code = torch.randint(-8, 8, (n, 1, d), generator=g).cuda()
        code[..., 0], code[..., 1] = -8, 7
        return torch.where(at < small, 0.0, a * u.double()).to(BF16), (code * torch.where(at < small, 1.0 / factor, 1.875)).to(BF16)
    c = Cache4([slots - 1], [1], H, 1, d, 64, rows=rows)
    c.q = u.to(BF16).expand(1, H, d).contiguous()
    return c


@pytest.mark.parametrize("d,H", [(128, 4), (64, 8), (128, 1)])
@pytest.mark.parametrize("slots,small,factor,score,full", [
    (768, 384, 2.0 ** 15, 7.9, False),      # a warp's second tile, 2^15.9 times as large
    (2304, 384, 2.0 ** 14, 7.9, True),      # 160 slots of a warp
    (8064, 384, 2.0 ** 14, 5.0, True),
    (32640, 384, 2.0 ** 13, 5.0, True),
    (130944, 384, 2.0 ** 9, 7.9, True),
    (130944, 384, 2.0 ** 60, 7.9, True),
    (8064, 384, 2.0 ** -40, 60.0, True),    # values that were large and count for little
    (8064, 4032, 1.0, 0.0, True)])
def test_values_that_grow_behind_a_warps_first_tile(slots, small, factor, score, full, d, H):
    """... in every warp of a step, of one sequence or of as many as the GPU has places for (which share their pages, so that a unit is one block's)."""
    c = grown(slots, small, factor, score, H, d)
    B = torch.cuda.get_device_properties(0).multi_processor_count if full else 1
    handle = glide.GlidePaged(c.k_pages, c.v_pages, H, B, c.slots, weights=False, head_dim=d)
    q = c.q.expand(B, H, d).contiguous()
    out, lse = torch.full_like(q, 7.0), torch.full((B, H), 7.0, device="cuda")
    handle.glide_paged_decode(c.table.expand(B, -1).contiguous(), c.lens_dev.expand(B).contiguous(), q, None, None, out, lse=lse)
    want, tol, want_lse, lse_tol = reference4(c)
    check(out, want.expand_as(q), tol.expand_as(q), "out")
    check(lse, want_lse.expand(B, H), lse_tol.expand(B, H), "lse")
    assert handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("of_q,of_k", [(2.0 ** 50, 2.0 ** 50), (2.0 ** 60, 2.0 ** 55), (2.0 ** 118, 2.0 ** -118), (2.0 ** -118, 2.0 ** 118), (2.0 ** -60, 2.0 ** -60)])
@pytest.mark.parametrize("d,H,Hkv", [(128, 4, 2), (64, 8, 1)])
def test_very_large_and_very_small_scores(of_q, of_k, d, H, Hkv):
    """Scores near 2^100 and 2^115, of which one slot takes all the weight; products that come out ordinary; scores of nothing."""
    c = Cache4([700, 5, 2000], [1, 1, 1], H, Hkv, d, 32, rows=lambda b, k, v: ((k.double() * of_k).to(BF16), v))
    c.q = (c.q.double() * of_q).to(BF16)
    out, lse = torch.full_like(c.q, 7.0), torch.full(c.q.shape[:2], 7.0, device="cuda")
    c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, None, None, out, lse=lse)
    want, tol, want_lse, lse_tol = reference4(c)
    check(out, want, tol, "out")
    check(lse, want_lse, lse_tol, "lse")
    assert c.handle.glide_paged_device_status() == 0
