"""Paged caches for the tests, and the definition of the paged operators in 64 bits, slot by slot (no code of the library)."""
import math

import torch

from paper_2607_24788_b200 import glide

BF16, F32 = torch.bfloat16, torch.float32


class Cache:
    """Pages, table and lengths of sequences that hold `before` slots and get `new` tokens.  Whatever no query may see (the
    rest of the pool, the slots behind a sequence) holds NaN, and the table's entries behind a sequence -1 and 2^30."""

    def __init__(self, before, new, heads, kv_heads, d, dtype, page, seed=0, layers=1, layout="hnd", amp=2.0, slots=None, weights=True):
        g = torch.Generator().manual_seed(seed)
        self.before, self.new, self.lens = list(before), list(new), [a + b for a, b in zip(before, new)]
        self.H, self.Hkv, self.G, self.d, self.dtype, self.page, self.L = heads, kv_heads, heads // kv_heads, d, dtype, page, layers
        B = len(self.lens)
        used = [-(-n // page) for n in self.lens]
        self.slots = slots or (max(used) + 1) * page
        cols, pages = -(-self.slots // page), sum(used) + 3
        ids = torch.randperm(pages, generator=g).tolist()
        table = torch.full((B, cols), -1, dtype=torch.int32)
        table[:, 1::2] = 1 << 30
        for b in range(B):
            table[b, :used[b]] = torch.tensor([ids.pop() for _ in range(used[b])], dtype=torch.int32)
        self.table_host, self.table = table, table.cuda()
        shape = (layers, pages, kv_heads, page, d) if layout == "hnd" else (layers, pages, page, kv_heads, d)
        self.k_pages, self.v_pages = (torch.full(shape, math.nan, dtype=dtype, device="cuda") for _ in range(2))
        if layout != "hnd":   # slots outside, heads inside
            self.k_pages, self.v_pages = self.k_pages.transpose(2, 3), self.v_pages.transpose(2, 3)
        T = sum(new)
        rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64).to(dtype)  # noqa: E731
        self.q, self.k, self.v = (rnd(T, heads, d).double() * amp).to(dtype).cuda(), rnd(T, kv_heads, d).cuda(), rnd(T, kv_heads, d).cuda()
        self.starts = torch.tensor([0] + list(new)).cumsum(0).to(torch.int32).cuda()
        self.lens_dev = torch.tensor(self.lens, dtype=torch.int32).cuda()
        # dense rows of every layer, sequence: [n][Hkv][d]
        self.dense = [[(rnd(n, kv_heads, d).cuda(), rnd(n, kv_heads, d).cuda()) for n in before] for _ in range(layers)]
        for l in range(layers):
            for b, n in enumerate(before):
                if n:
                    page_of, off = self.place(b, torch.arange(n, device="cuda"))
                    self.k_pages[l][page_of, :, off], self.v_pages[l][page_of, :, off] = self.dense[l][b]
        self.weights_kept = weights
        self.weight = torch.rand((B, kv_heads, self.slots), generator=g).cuda()
        self.pos = torch.randint(0, 1 << 20, (B, kv_heads, self.slots), generator=g, dtype=torch.int32).cuda()
        self.handle = glide.GlidePaged(self.k_pages, self.v_pages, heads, B, self.slots, weights=weights)

    def place(self, b, slot):
        return self.table[b, slot // self.page].long(), slot % self.page

    def rows(self, l, b):
        """K, V of sequence b as they should stand in the cache once the new tokens are stored: [n][Hkv][d]."""
        s = slice(int(self.starts[b]), int(self.starts[b + 1]))
        return tuple(torch.cat([old, new[s]]) for old, new in zip(self.dense[l][b], (self.k, self.v)))

    def expect_pages(self, l=0, stored=True):
        """Pools in which every slot holds its row and everything else what it held at the start (NaN)."""
        want = [torch.full_like(self.k_pages[l], math.nan), torch.full_like(self.v_pages[l], math.nan)]
        for b, n in enumerate(self.lens):
            n = n if stored else self.before[b]
            if n:
                page_of, off = self.place(b, torch.arange(n, device="cuda"))
                for w, r in zip(want, self.rows(l, b)):
                    w[page_of, :, off] = r[:n]
        return want

    def check_pages(self, l=0, stored=True):
        for got, want in zip((self.k_pages[l], self.v_pages[l]), self.expect_pages(l, stored)):
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


def reference(c, window=-1, n_sink=0, layer=0, scale=None, rounded=None):
    """Outputs [T][H][d], lse [T][H], the weights given to every slot [B][Hkv][slots], all fp64, and how far an implementation
    may be off them.  Bounds, with u = 2^-24 (fp32) and A the largest sum_k |q_k k_jk| scale of a row's slots:
      a score is off by at most e = (d + 4) 2u A (products and sums of d terms, tensor cores may cut off instead of rounding), the
      reference subtracted from it by 4u A more, 2^x by 4u relative; so every weight by w = 2 (e + 8u A) + 16u + n 2u (its own and the row
      sum's, whose n terms are summed in fp32), relative
      outputs: sum_j p_j |v_j - o| (w + r) + 2u (n + 4) sum_j p_j |v_j| + the rounding of o, with r = 2^-8 (bf16 weights in the product)
      lse: e + 8u A + 8u + n 2u + 2u |lse|;  weights: sum of the terms' w, and one rounding per term and of the sum; a term below
      the least normal number, 2^-126, may be 0"""
    u = 2.0 ** -24
    d, G = c.d, c.G
    scale = d ** -0.5 if scale is None else scale
    out = torch.zeros(c.q.shape, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    lse = torch.full(c.q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    lse_tol = torch.zeros_like(lse)
    given = torch.zeros(c.weight.shape, dtype=torch.float64, device="cuda")
    given_tol = torch.zeros_like(given)
    half = torch.finfo(c.dtype).eps / 2
    r = half if c.dtype is BF16 else 0.0
    for b, n in enumerate(c.lens):
        T, row = c.new[b], int(c.starts[b])
        if not T:
            continue
        keys, values = (x.double() for x in c.rows(layer, b))
        i = torch.arange(n - T, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None]
        sees = (j <= i) & ((j > i - window) | (j < n_sink) if window >= 0 else torch.ones_like(j > i))
        cnt = sees.sum(1).double()
        for h in range(c.H):
            q, k, v = c.q[row:row + T, h].double(), keys[:, h // G], values[:, h // G]
            s = torch.where(sees, q @ k.T * scale, -math.inf)
            A = torch.where(sees, q.abs() @ k.abs().T * scale, 0.0).amax(1)
            total = torch.logsumexp(s, 1)
            p = torch.where(sees, torch.exp(s - torch.where(total == -math.inf, 0.0, total)[:, None]), 0.0)
            o = p @ v
            e = (d + 4) * 2 * u * A + 8 * u * A
            w = 2 * e + 16 * u + cnt * 2 * u
            spread = (p[:, :, None] * (v[None] - o[:, None]).abs()).sum(1)
            out[row:row + T, h] = o
            tol[row:row + T, h] = spread * (w + r)[:, None] + 2 * u * (cnt + 4)[:, None] * (p @ v.abs()) + half * o.abs() * (1 + 2 * r) + 1e-30
            lse[row:row + T, h] = total
            lse_tol[row:row + T, h] = e + 8 * u + cnt * 2 * u + 2 * u * total.abs().nan_to_num(posinf=0.0)
            given[b, h // G, :n] += p.sum(0)
            given_tol[b, h // G, :n] += (p * (w + u * (T * G + 2))[:, None]).sum(0) + T * 2.0 ** -126
    return out, tol, lse, lse_tol, given, given_tol


def check(got, want, tol, what):
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN where there should be none, or the other way round"
    off = (got - want).abs()
    same = torch.isinf(want) & (got == want) | want.isnan()
    bad = ~same & ~(off <= tol)
    if bad.any():
        at = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: {got[at]} against {want[at]}, may be off by {tol[at]}")
