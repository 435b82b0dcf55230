"""Sparse steps whose border lies among pages of almost the same score, which only sums in 64 bits tell apart, wherever among the columns they stand."""
import pytest
import torch

from tests.paged_more_util import choose, page_scores
from tests.paged_util import BF16, Cache
from tests.test_gpu_paged_sparse import Sparse
from tests.test_gpu_paged_sparse_close import with_keys

pytestmark = pytest.mark.gpu


def border_cache(pages, near, high, H, Hkv, d, seed=0):
    """One key for all slots of a page: `near` pages whose scores differ in the last feature only, `high` ones of twice the score, the others of a
    quarter of it."""
    g = torch.Generator().manual_seed(seed)
    u = torch.randint(0, 2, (Hkv, d), generator=g).double().cuda() * 2 - 1

    def make(k):
        s = torch.full((pages,), 0.25, dtype=torch.float64, device="cuda")
        s[near], s[high] = 1.0, 2.0
        key = s[:, None, None] * u
        key[:, :, -1] = torch.randn((pages, Hkv), generator=g, dtype=torch.float64).cuda() * 2.0 ** -12
        return key.repeat_interleave(16, 0).to(BF16)
    c = with_keys(Cache([16 * pages], [1], H, Hkv, d, BF16, 16, seed=seed), make)
    c.q = (c.q.double().abs() * u.repeat_interleave(H // Hkv, 0)).to(BF16)
    return c


@pytest.mark.parametrize("pages", [300, 2050, 2300])
@pytest.mark.parametrize("n_near", [10, 100, 200])
@pytest.mark.parametrize("where", ["first", "last", "spread"])
def test_the_choice_does_not_depend_on_timing(pages, n_near, where):
    """Some warps have keys of the border in their runs, others have none, or shorter runs: the choice is the definition's, every time."""
    near = {"first": torch.arange(n_near), "last": torch.arange(pages - n_near, pages), "spread": torch.arange(n_near) * (pages // n_near)}[where]
    high = [i for i in range(pages // 2, pages) if i not in set(near.tolist())][:30]
    c = border_cache(pages, near.cuda(), torch.tensor(high, dtype=torch.long).cuda(), 2, 2, 64)
    s = Sparse(c, 1 + len(high) + n_near // 2)
    s.step(c.k, c.v)
    s.check()
    scores = page_scores(c.q[0], s.bounds, c.table[0], pages + 1)
    want = torch.tensor([choose(scores[g], s.n_picks, 16, 0) for g in range(2)], dtype=torch.int32, device="cuda")
    all_picks = []
    for _ in range(40):
        s.step(c.k, c.v)
        all_picks.append(s.picks[0].clone())
    assert all(torch.equal(p, want) for p in all_picks)


@pytest.mark.parametrize("d,H", [(128, 1), (128, 8), (64, 2)])
@pytest.mark.parametrize("below", [22, 23, 24, 25, 26])
def test_sums_that_lose_what_an_adder_can(d, H, below):
    """One large product and others just below 2^-below of it, which an adder of so many bits cuts off one by one: the choice is that of sums in 64 bits.  The bound
    that a score goes by (beside it in the work space: bits of a float above those of the score in order) covers what 2 d additions of 23 bits can lose."""
    pages = 300
    g = torch.Generator().manual_seed(below)
    at = torch.arange(pages)

    def make(k):
        key = torch.full((pages, 1, d), (2 - 2.0 ** -7) * 2.0 ** -below, dtype=torch.float64)
        key[torch.rand((pages, 1, d), generator=g) < 0.2] = 0.0
        key[at, 0, at % d] = 1.0
        return key.repeat_interleave(16, 0).to(BF16).cuda()
    c = with_keys(Cache([16 * pages], [1], H, 1, d, BF16, 16), make)
    c.q = torch.ones_like(c.q)
    c.q[:, 1::2] = 0.5
    s = Sparse(c, 40)
    s.step(c.k, c.v)
    s.check()
    key = s.scores.view(torch.int64)[0, 0, :pages]
    order, err = key & 0xffffffff, (key >> 32).to(torch.int32).view(torch.float32).double()
    bits = torch.where(order >= 1 << 31, order - (1 << 31), 0xffffffff - order)
    got = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).to(torch.int32).view(torch.float32).double()
    want = page_scores(c.q[0], s.bounds, c.table[0], pages)[0]   # (of numbers that are not negative: their absolute values' sum too)
    assert ((got - want).abs() <= err).all()
    assert (err >= 2 * d * 2.0 ** -23 * want).all()
