"""Prompts whose weights spread over many powers of two: over a cache in 4 bits small ones are not lost beside a large one; no row loses all of them."""
import math

import pytest
import torch

from tests.paged_more_util import BF16, Cache4, levels, reference4
from tests.paged_util import Cache, check, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,H,before,new", [(64, 1, 122872, 8200), (128, 8, 129972, 1100)])
@pytest.mark.parametrize("first", [25.5, 20.0, 27.0])
def test_a_first_token_that_takes_most_of_a_prompts_weight(d, H, before, new, first):
    """The first slot has 2^first of every other one's weight and a value of 0, all others the value 1: slot i's output is i / (i + 2^first).  Weights are
    fp16 numbers, the largest one at least 2^5: each is off by 2^-11 of itself or by 2^-25, 2^-30 of the largest; outputs are rounded to bf16.  (As
    many rows as here are not cut into parts.)"""
    u = torch.ones(d, dtype=torch.float64, device="cuda")
    u[1::3] = -1.0

    def rows(b, k, v):
        k, v = torch.zeros_like(k), torch.ones_like(v)
        k[0], v[0] = (first * math.log(2.0) / d ** 0.5 * u).to(BF16), 0.0
        return k, v
    c = Cache4([before], [new], H, 1, d, 64, rows=rows)
    c.q = u.to(BF16).expand(new, H, d).contiguous()
    out, lse = torch.full_like(c.q, 7.0), torch.full((new, H), 7.0, device="cuda")
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, None, None, out, lse=lse)
    code, step, low = levels(c.rows(0, 0)[0][0, 0])
    x = (u * (code.double() * step.double() + low.double())).sum() * d ** -0.5
    i = torch.arange(before, before + new, dtype=torch.float64, device="cuda")[:, None, None]
    want = (i / (i + x.exp())).expand(c.q.shape)
    # the score: as tests/paged_more_util.py has it for prompts, with Q = d^0.5, steps and middle levels of the one key that is not 0
    U, Q = 2.0 ** -24, d ** 0.5
    mid = (low.double() + 8 * step.double()).abs()
    e = Q * ((d + 8) * 2 * U * (8 * step.double() + mid) + 2.0 ** -20 * mid) + d * 2.0 ** -31 * d ** -0.5 * (8 * step.double() + mid)
    n = before + new
    w = 2 * (e + 8 * U * x) + 16 * U + n * 2 * U
    tol = want * (w + 2.0 ** -11 + 2.0 ** -8 * (1 + 2.0 ** -7)) + n * 2.0 ** -30
    check(out, want, tol, "out")
    total = (i + x.exp()).log().squeeze(2)
    check(lse, total.expand(new, H), (e + 8 * U * x + 8 * U + n * 2 * U + 2 * U * total).expand(new, H), "lse")
    assert c.handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("of_q,of_k", [(2.0 ** 14, 2.0 ** 14), (2.0 ** 16, 2.0 ** 15), (2.0 ** 50, 2.0 ** 50), (2.0 ** 60, 2.0 ** 50), (2.0 ** -60, 2.0 ** -60)])
@pytest.mark.parametrize("d,H,Hkv,before,new", [(128, 4, 2, [700, 0], [40, 130]), (64, 8, 1, [9000], [5])])
def test_scores_beyond_what_a_reference_can_hold(codes, of_q, of_k, d, H, Hkv, before, new):
    """Scores so large that a number next to the largest one is whole powers of two away: one slot takes all the weight, and none is lost.  In tiles and in
    parts of the key tiles."""
    scaled = lambda x, f: (x.double() * f).to(BF16)  # noqa: E731
    if codes:
        c = Cache4(before, new, H, Hkv, d, 32, rows=lambda b, k, v: (scaled(k, of_k), v))
    else:
        c = Cache(before, new, H, Hkv, d, BF16, 32)
        c.dense = [[(scaled(k, of_k), v) for k, v in rows] for rows in c.dense]
        c.k = scaled(c.k, of_k)
        for b, n in enumerate(c.lens):
            at, off = c.place(b, torch.arange(n, device="cuda"))
            for pool, x in zip((c.k_pages, c.v_pages), c.rows(0, b)):
                pool[0][at, :, off] = x
    c.q = scaled(c.q, of_q)
    out, lse = torch.full_like(c.q, 7.0), torch.full(c.q.shape[:2], 7.0, device="cuda")
    for with_lse in (lse, None):
        c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, None, None, out, lse=with_lse)
        want, tol, want_lse, lse_tol = (reference4(c, prompt=True) if codes else reference(c))[:4]
        check(out, want, tol, "out")
    check(lse, want_lse, lse_tol, "lse")
    assert c.handle.glide_paged_device_status() == 0
