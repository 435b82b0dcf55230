"""Steps over selected pages: which pages are chosen, and the attention over them, against the definitions in 64 bits; the operators in a row."""
import math

import pytest
import torch

from paper_2607_24788_b200 import glide
from tests.paged_more_util import BF16, U, Cache4, angles, choose, page_scores, reference4, rotate
from tests.paged_util import F32, Cache, check, reference

pytestmark = pytest.mark.gpu


class Sparse:
    def __init__(self, c, n_picks, n_sink=0, fresh=True):
        self.c, self.n_picks, self.n_sink = c, n_picks, n_sink
        B = len(c.lens)
        self.bounds = torch.full((c.k_pages.shape[1], c.Hkv, 2, c.d), 7.0, dtype=c.dtype, device="cuda")
        for b, n in enumerate(c.before):
            for col in range(-(-n // c.page)):
                x = c.dense[0][b][0][col * c.page:(col + 1) * c.page]
                self.bounds[int(c.table[b, col])] = torch.stack([x.amin(0), x.amax(0)], 1)
        self.picks = torch.full((B, c.Hkv, n_picks), 99, dtype=torch.int32, device="cuda")
        self.scores = torch.empty((B, c.Hkv, c.table.shape[1]), dtype=torch.float64, device="cuda")
        self.out, self.lse = torch.full_like(c.q, 7.0), torch.full(c.q.shape[:2], 7.0, device="cuda")

    def step(self, k, v, **kw):
        c = self.c
        c.handle.glide_paged_decode_sparse(c.table, c.lens_dev, c.q, k, v, self.out, self.bounds, self.picks, self.scores, lse=self.lse, n_sink=self.n_sink, **kw)

    def check(self):
        """Picks and bounds equal the definition's; outputs as the dense step's over the picked slots, by its bounds."""
        c = self.c
        want_bounds = self.bounds.clone()
        for b, n in enumerate(c.lens):
            if n:
                x = c.rows(0, b)[0][(n - 1) // c.page * c.page:]
                want_bounds[int(c.table[b, (n - 1) // c.page])] = torch.stack([x.amin(0), x.amax(0)], 1)
        assert torch.equal(self.bounds.isnan(), want_bounds.isnan()) and torch.equal(self.bounds.nan_to_num(), want_bounds.nan_to_num())
        for b, n in enumerate(c.lens):
            pages = -(-n // c.page)
            scores = page_scores(c.q[b], self.bounds, c.table[b], pages) if n else None
            for g in range(c.Hkv):
                want = choose(scores[g], self.n_picks, c.page, self.n_sink) if n else []
                assert self.picks[b, g].tolist() == want + [-1] * (self.n_picks - len(want)), (b, g)
                heads = slice(g * c.G, (g + 1) * c.G)
                if not n:
                    assert not self.out[b, heads].any() and (self.lse[b, heads] == -math.inf).all()
                    continue
                slots = torch.cat([torch.arange(i * c.page, min(n, (i + 1) * c.page)) for i in want]).cuda()
                k, v = (x[slots, g].double() for x in c.rows(0, b))
                q = c.q[b, heads].double()
                x = q @ k.T * c.d ** -0.5
                A = (q.abs() @ k.abs().T).amax(1) * c.d ** -0.5
                total = torch.logsumexp(x, 1)
                p = torch.exp(x - total[:, None])
                o = p @ v
                cnt, half = len(slots), torch.finfo(c.dtype).eps / 2
                e = (c.d + 4) * 2 * U * A + 8 * U * A
                w = 2 * e + 16 * U + cnt * 2 * U + (half if c.dtype is BF16 else 0.0)
                tol = (p[:, :, None] * (v[None] - o[:, None]).abs()).sum(1) * w[:, None] + 2 * U * (cnt + 4) * (p @ v.abs()) + half * o.abs() * (1 + 2 * half) + 1e-30
                check(self.out[b, heads], o, tol, f"out {b} {g}")
                check(self.lse[b, heads], total, e + 8 * U + cnt * 2 * U + 2 * U * total.abs(), f"lse {b} {g}")
        assert c.handle.glide_paged_device_status() == 0


SHAPES = [(F32, 64, 4, 4, 16), (F32, 128, 8, 1, 32), (BF16, 128, 32, 8, 64), (BF16, 64, 6, 6, 16), (BF16, 128, 8, 1, 128), (BF16, 64, 4, 2, 32)]


@pytest.mark.parametrize("dtype,d,H,Hkv,page", SHAPES)
@pytest.mark.parametrize("n_picks,n_sink", [(1, 0), (2, 1), (3, 0), (7, 20), (40, 4), (500, 0)])
def test_sparse_step(dtype, d, H, Hkv, page, n_picks, n_sink):
    if -(-n_sink // page) + 1 > n_picks:
        n_sink = 1
    lens = [1, 2, page, page + 1, 5 * page, 40 * page - 3, 700, 1500]
    c = Cache([n - 1 for n in lens], [1] * len(lens), H, Hkv, d, dtype, page)
    s = Sparse(c, n_picks, n_sink)
    s.step(c.k, c.v, pos=c.pos)
    s.check()
    c.check_pages()
    assert all((c.pos[b, :, n - 1] == n - 1).all() for b, n in enumerate(lens))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_sequences_and_more_pages_than_threads(dtype):
    c = Cache([30000, 9001, 0], [1, 1, 1], 4, 2, 64, dtype, 16)
    s = Sparse(c, 600, 4)
    s.step(c.k, c.v)
    s.check()
    c = Cache([40000], [1], 8, 1, 128, dtype, 16)
    s = Sparse(c, 33)
    s.step(c.k, c.v)
    s.check()


def test_equal_scores_and_zeros():
    """Pages with the same bounds: the first ones; all of them; zeros of either sign."""
    for make in (lambda x: x * 0.0, lambda x: -x * 0.0, lambda x: x[:16].repeat(len(x) // 16 + 1, 1, 1)[:len(x)]):
        c = Cache([800], [1], 4, 2, 64, BF16, 16)
        k, v = c.dense[0][0]
        k = make(k)
        c.dense[0][0] = (k, v)
        at, off = c.place(0, torch.arange(800, device="cuda"))
        c.k_pages[0][at, :, off] = k
        s = Sparse(c, 10, 1)
        s.step(c.k, c.v)
        s.check()
        assert (s.picks[0, :, :9] == torch.arange(9, device="cuda")).all() and (s.picks[0, :, 9] == 50).all()


def test_scores_that_are_no_numbers():
    """A NaN or an infinity among a page's keys: its score counts as the largest, in every KV head by itself."""
    c = Cache([800], [1], 4, 2, 64, BF16, 16)
    k, v = c.dense[0][0]
    k[16 * 30 + 2, 0, 7], k[16 * 31, 1, 9], k[16 * 33 + 5, 1, 3] = math.nan, math.inf, math.nan
    at, off = c.place(0, torch.arange(800, device="cuda"))
    c.k_pages[0][at, :, off] = k
    s = Sparse(c, 4)
    s.step(c.k, c.v)
    scores = page_scores(c.q[0], s.bounds, c.table[0], 51)
    for g in range(2):
        assert s.picks[0, g].tolist() == choose(scores[g], 4, 16, 0)
    assert 30 in s.picks[0, 0].tolist() and 33 in s.picks[0, 1].tolist() and 31 in s.picks[0, 1].tolist()
    assert s.out[0, :2].isnan().all() and s.out[0, 2:].isnan().all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_an_empty_sequence_and_tokens_in_the_cache(dtype):
    c = Cache([500, 0, 64], [1, 0, 1], 4, 2, 64, dtype, 16)
    c.q, c.k, c.v = (torch.cat([x[:1], x[:1] * math.nan, x[1:]]) for x in (c.q, c.k, c.v))
    c.starts = torch.tensor([0, 1, 1, 2], dtype=torch.int32, device="cuda")
    c.handle.glide_paged_append(c.table, c.lens_dev, None, None, c.k, c.v)
    c.k, c.v = c.k[[0, 2]], c.v[[0, 2]]
    s = Sparse(c, 5, 3)
    s.step(None, None)
    s.check()


def test_replayed_with_other_lengths():
    c = Cache([1999, 100], [1, 1], 4, 2, 64, BF16, 16)
    s = Sparse(c, 8, 1)
    s.step(c.k, c.v)
    s.check()
    lens, want = c.lens_dev, (s.out.clone(), s.picks.clone())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s.step(c.k, c.v)
    for n in ((2000, 101), (40, 5), (2000, 101)):
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        if n[0] == 2000:
            graph.replay()
            assert torch.equal(s.out, want[0]) and torch.equal(s.picks, want[1])
        else:
            k_pages, v_pages, bounds = c.k_pages.clone(), c.v_pages.clone(), s.bounds.clone()
            graph.replay()
            assert (s.picks[:, :, 4:] == -1).all() and (s.picks[0, :, :3] == torch.arange(3, device="cuda")).all()
            c.k_pages.copy_(k_pages), c.v_pages.copy_(v_pages), s.bounds.copy_(bounds)
    assert c.handle.glide_paged_device_status() == 0


def test_a_prompt_then_sparse_steps():
    """As they are used together: a prompt comes in rotated and attends, its bounds are made, steps over selected pages follow."""
    B, H, Hkv, d, page, steps = 2, 8, 2, 64, 16, 20
    c = Cache([0] * B, [200, 131], H, Hkv, d, BF16, page, slots=256)
    cos, sin = angles(400, d)
    turn = glide.GlideRotation(cos, sin)
    ids = torch.randperm(40)[:32].to(torch.int32).view(2, 16)
    c.table = ids.cuda()
    c.k_pages, c.v_pages = (torch.full((1, 40, Hkv, page, d), math.nan, dtype=BF16, device="cuda") for _ in range(2))
    c.handle = glide.GlidePaged(c.k_pages, c.v_pages, H, B, 256, weights=False)
    q = torch.empty_like(c.q)
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, q, rotation=turn)
    bounds = torch.empty((40, Hkv, 2, d), dtype=BF16, device="cuda")
    c.handle.glide_paged_bounds(c.table, c.lens_dev, c.starts, bounds)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, q, None, None, out, lse=lse)
    p = torch.cat([torch.arange(n) for n in c.lens]).cuda()
    c.q, c.k = rotate(c.q, cos, sin, p, False), rotate(c.k, cos, sin, p, False)
    want, tol, want_lse, lse_tol = reference(c)[:4]
    check(out, want, tol, "out")
    check(lse, want_lse, lse_tol, "lse")
    rows = [c.rows(0, b) for b in range(B)]
    g = torch.Generator().manual_seed(5)
    for i in range(steps):
        q1, k1, v1 = (torch.randn((B, h, d), generator=g).to(BF16).cuda() * 2 for h in (H, Hkv, Hkv))
        lens = torch.tensor([n + 1 for n in c.lens], dtype=torch.int32, device="cuda")
        turned = torch.empty_like(q1)
        c.handle.glide_paged_append(c.table, lens, None, q1, k1, v1, turned, rotation=turn)
        at = lens.long() - 1
        step = Cache.__new__(Cache)
        step.__dict__.update(c.__dict__)
        step.before, step.new, step.lens, step.lens_dev = c.lens, [1, 1], [n + 1 for n in c.lens], lens
        step.dense, step.starts = [rows], torch.arange(3, dtype=torch.int32, device="cuda")
        step.q, step.k, step.v = rotate(q1, cos, sin, at, False), rotate(k1, cos, sin, at, False), v1
        assert torch.equal(turned, step.q)
        s = Sparse(step, 6, 2)
        s.bounds = bounds
        s.step(None, None)
        s.check()
        rows = [step.rows(0, b) for b in range(B)]
        c.lens = step.lens


def test_a_prompt_then_steps_in_4_bits():
    """The same over pages in 4 bits: append, attend, a further turn, steps."""
    c = Cache4([0, 0], [150, 301], 8, 2, 128, 32, stored=False)
    cos, sin = angles(400, 128)
    turn = glide.GlideRotation(cos, sin, neighbours=True)
    q, out = torch.empty_like(c.q), torch.empty_like(c.q)
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, q, rotation=turn)
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, q, None, None, out)
    p = torch.cat([torch.arange(n) for n in c.lens]).cuda()
    c.q, c.k = rotate(c.q, cos, sin, p, True), rotate(c.k, cos, sin, p, True)
    assert torch.equal(q, c.q)
    c.check_pages()
    check(out, *reference4(c, prompt=True)[:2], "out")
    g = torch.Generator().manual_seed(5)
    for i in range(5):
        q1, k1, v1 = (torch.randn((2, h, 128), generator=g).to(BF16).cuda() for h in (8, 2, 2))
        c.dense = [[c.rows(0, b) for b in range(2)]]
        c.before, c.new, c.lens = c.lens, [1, 1], [n + 1 for n in c.lens]
        c.starts, c.lens_dev = torch.arange(3, dtype=torch.int32, device="cuda"), torch.tensor(c.lens, dtype=torch.int32, device="cuda")
        out = torch.empty_like(q1)
        c.handle.glide_paged_append(c.table, c.lens_dev, None, q1, k1, v1, q1, rotation=turn)
        c.handle.glide_paged_decode(c.table, c.lens_dev, q1, None, None, out)
        c.q, c.v = q1, v1
        c.k = rotate(k1, cos, sin, c.lens_dev.long() - 1, True)
        check(out, *reference4(c)[:2], "out")
        c.check_pages()
    assert c.handle.glide_paged_device_status() == 0
