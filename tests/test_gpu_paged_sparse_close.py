"""Sparse steps whose pages' scores lie so close together, or are so large, small or many, that sums of 32 bits would not tell them apart."""
import math

import pytest
import torch

from tests.paged_util import BF16, F32, Cache
from tests.test_gpu_paged_sparse import Sparse

pytestmark = pytest.mark.gpu


def with_keys(c, make):
    """The cache's old keys become make(keys [n][Hkv][d])."""
    n = c.before[0]
    k, v = c.dense[0][0]
    k = make(k)
    c.dense[0][0] = (k, v)
    at, off = c.place(0, torch.arange(n, device="cuda"))
    c.k_pages[0][at, :, off] = k
    return c


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pages", [60, 300, 3000])
@pytest.mark.parametrize("n_picks", [5, 48])
def test_scores_next_to_each_other(dtype, pages, n_picks):
    """Every page has one of four keys, but for the last feature of the smallest weight: thousands of scores within a rounding of each other."""
    def make(k):
        same = k[:4].repeat(len(k) // 4 + 1, 1, 1)[:len(k)].view(-1, 16, *k.shape[1:])[:, :1].repeat(1, 16, 1, 1).flatten(0, 1).clone()
        same[:, :, -1] = k[:, :, -1] * 2.0 ** -12
        return same
    c = with_keys(Cache([16 * pages], [1], 8, 2, 64, dtype, 16), make)
    s = Sparse(c, n_picks, 1)
    s.step(c.k, c.v)
    s.check()


@pytest.mark.parametrize("of_q,of_k", [(2.0 ** -70, 2.0 ** -70), (2.0 ** 60, 2.0 ** 66), (2.0 ** -100, 2.0 ** 100)])
def test_very_small_and_very_large_scores(of_q, of_k):
    c = Cache([1600], [1], 4, 1, 128, BF16, 16)
    c.q = (c.q.double() * of_q).to(BF16)
    with_keys(c, lambda k: (k.double() * of_k).to(BF16))
    c.k = (c.k.double() * of_k).to(BF16)
    s = Sparse(c, 20, 1)
    c.handle.glide_paged_decode_sparse(c.table, c.lens_dev, c.q, c.k, c.v, s.out, s.bounds, s.picks, s.scores, n_sink=1)
    from tests.paged_more_util import choose, page_scores
    scores = page_scores(c.q[0], s.bounds, c.table[0], 101)
    assert s.picks[0, 0].tolist() == choose(scores[0], 20, 16, 1)
    assert c.handle.glide_paged_device_status() == 0


def test_an_odd_query():
    """A query that is no number: every score is NaN, the first pages are taken."""
    c = Cache([800, 800], [1, 1], 4, 2, 64, BF16, 16)
    c.q[0, 1, 3], c.q[1, 3, 0] = math.nan, math.inf
    s = Sparse(c, 7)
    s.step(c.k, c.v)
    assert s.picks[0, 0].tolist() == [0, 1, 2, 3, 4, 5, 50]
    from tests.paged_more_util import choose, page_scores
    for b in range(2):
        scores = page_scores(c.q[b], s.bounds, c.table[b], 51)
        for g in range(2):
            assert s.picks[b, g].tolist() == choose(scores[g], 7, 16, 0)
