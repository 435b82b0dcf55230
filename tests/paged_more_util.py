"""Pages in 4 bits for the tests, the rotation and the scores of pages, from their definitions (no code of the library)."""
import math

import torch

from paper_2607_24788_b200 import glide

BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def levels(x):
    """Codes, step and lowest level of bf16 rows [.., d]; a row that is not finite stands for NaN."""
    x = x.float()
    low, high = x.amin(-1), x.amax(-1)
    step = ((high - low) * torch.tensor(1.0 / 15.0, dtype=F32, device=x.device)).to(BF16).float()
    bad = ~(x.isfinite().all(-1) & step.isfinite())
    code = torch.where(step[..., None] > 0, ((x - low[..., None]) / step[..., None]).round().clamp(0, 15), 0.0)
    code = torch.where(bad[..., None], 0.0, code)
    return code.to(torch.uint8), torch.where(bad, math.nan, step), torch.where(bad, math.nan, low)


def pack_row(code, step, low):
    """The bytes of rows: codes [.., d / 2], levels [.., 4]."""
    both = torch.stack([step, low], -1).to(BF16).contiguous().view(torch.int16)
    return code[..., 0::2] | code[..., 1::2] << 4, torch.where(step.isnan()[..., None], 0x7fc0, both).to(torch.int16).view(torch.uint8)   # (one NaN)


class Cache4:
    """Sequences that hold `before` slots and get `new` tokens, in pages of 4 bits.  The rest of the pool holds bytes of 0xff: codes of 15 and NaN
    for levels; the table's entries behind a sequence are -1 and 2^30.  amp: of the queries; scale(l, b) a factor of the values."""

    def __init__(self, before, new, heads, kv_heads, d, page, seed=0, layers=1, amp=2.0, gap=0, stored=True, rows=None):
        g = torch.Generator().manual_seed(seed)
        self.before, self.new, self.lens = list(before), list(new), [a + b for a, b in zip(before, new)]
        self.H, self.Hkv, self.G, self.d, self.page, self.L = heads, kv_heads, heads // kv_heads, d, page, layers
        B = len(self.lens)
        used = [-(-n // page) for n in self.lens]
        self.slots = (max(used) + 1) * page
        cols, pages = max(used) + 1, sum(used) + 3
        ids = torch.randperm(pages, generator=g).tolist()
        table = torch.full((B, cols), -1, dtype=torch.int32)
        table[:, 1::2] = 1 << 30
        for b in range(B):
            table[b, :used[b]] = torch.tensor([ids.pop() for _ in range(used[b])], dtype=torch.int32)
        self.table = table.cuda()
        self.row_bytes = glide.paged4_row_bytes(d)
        block = page * self.row_bytes
        self.k_pages, self.v_pages = (torch.full((layers, pages, kv_heads, block + gap), 255, dtype=torch.uint8, device="cuda")[..., :block] for _ in range(2))
        T = sum(new)
        rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64).to(BF16).cuda()  # noqa: E731
        self.q, self.k, self.v = (rnd(T, heads, d).double() * amp).to(BF16), rnd(T, kv_heads, d), rnd(T, kv_heads, d)
        self.starts = torch.tensor([0] + list(new)).cumsum(0).to(torch.int32).cuda()
        self.lens_dev = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.dense = [[(rnd(n, kv_heads, d), rnd(n, kv_heads, d)) for n in before] for _ in range(layers)]
        if rows is not None:   # (changes the rows, [n][Hkv][d] of K and of V of a sequence, old and new together)
            for l in range(layers):
                for b in range(B):
                    k, v = rows(b, *self.rows(l, b))
                    n, s = self.before[b], slice(int(self.starts[b]), int(self.starts[b + 1]))
                    self.dense[l][b] = (k[:n], v[:n])
                    self.k[s], self.v[s] = k[n:], v[n:]
        for l in range(layers):
            for b in range(B):
                self.put(l, b, self.lens[b] if stored else self.before[b])
        self.handle = glide.GlidePaged(self.k_pages, self.v_pages, heads, B, self.slots, weights=False, head_dim=d)

    def rows(self, l, b):
        s = slice(int(self.starts[b]), int(self.starts[b + 1]))
        return tuple(torch.cat([old, new[s]]) for old, new in zip(self.dense[l][b], (self.k, self.v)))

    def put(self, l, b, n, pools=None):
        """The first n rows of sequence b into the pools (default: the cache's own)."""
        if not n:
            return
        slot = torch.arange(n, device="cuda")
        page, off = self.table[b, slot // self.page].long(), slot % self.page
        for pool, x in zip(pools or (self.k_pages[l], self.v_pages[l]), self.rows(l, b)):
            codes, lev = pack_row(*levels(x[:n]))
            blocks = pool[..., :self.page * self.row_bytes]
            head = torch.arange(self.Hkv, device="cuda")[:, None]
            half = self.d // 2
            blocks[page[:, None, None], head, (off * half)[:, None, None] + torch.arange(half, device="cuda")] = codes
            blocks[page[:, None, None], head, (self.page * half + off * 4)[:, None, None] + torch.arange(4, device="cuda")] = lev

    def expect_pages(self, l=0):
        want = [torch.full_like(self.k_pages[l], 255), torch.full_like(self.v_pages[l], 255)]
        for b, n in enumerate(self.lens):
            self.put(l, b, n, want)
        return want

    def check_pages(self, l=0):
        for got, want in zip((self.k_pages[l], self.v_pages[l]), self.expect_pages(l)):
            assert torch.equal(got, want)

    def values(self, l, b):
        """What the rows of sequence b stand for, fp64 [n][Hkv][d] of K and V, and their steps and lowest levels [n][Hkv]."""
        out = []
        for x in self.rows(l, b):
            code, step, low = levels(x)
            out.append((code.double() * step.double()[..., None] + low.double()[..., None], step.double(), low.double()))
        return out


def reference4(c, window=-1, n_sink=0, layer=0, prompt=False):
    """Outputs and lse in fp64 and how far an implementation may be off them, with u = 2^-24, s the step, m = low + 8 s the middle level, n = code - 8,
    Q = sum |q|, all times the softmax scale:
      a step of one token: codes against q in fp32 on tensor cores, which may cut off: e = (d + 8) 2u Q (15 s + |low|);
        weights times step are rounded to bf16: 2^-8 sum p |v - m|
      prompts: e = (d + 8) 2u Q (8 s + |m|) + 2^-20 Q |m| (two numbers of 22 bits) + d 2^-31 max|q| max|k| (queries below 2^-20 of a row's largest), and
        2^-19 Q max|k| for rows whose step is below 2^-8 of the largest key; weights rounded to fp16: 2^-11 sum p |v| + cnt 2^-25 max|v|; values:
        sum p max(2^-11 |v|, 2^-16 max|v|)
      a weight is off by w = 2 (e + 8u |x|) + 16u + cnt 2u of itself (its own and the sum's), outputs by sum p |v - o| w, by 2u (cnt + 8) sum p (|v - m| + |m|)
      of the sums, and by their rounding, 2^-8 |o|;  lse: e + 8u |x| + 8u + cnt 2u + 2u |lse|, where x are the scores seen."""
    d, G, scale = c.d, c.G, c.d ** -0.5
    out = torch.zeros(c.q.shape, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    lse = torch.full(c.q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    lse_tol = torch.zeros_like(lse)
    for b, n in enumerate(c.lens):
        T, row = c.new[b], int(c.starts[b])
        if not T or not n:
            continue
        (keys, ks, kl), (values, vs, vl) = c.values(layer, b)
        i = torch.arange(n - T, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None]
        sees = (j <= i) & ((j > i - window) | (j < n_sink) if window >= 0 else torch.ones_like(j > i))
        cnt = sees.sum(1).double()
        fine = lambda x: torch.where(x.isfinite(), x, 0.0)  # noqa: E731
        for h in range(c.H):
            g = h // G
            q, k, v = c.q[row:row + T, h].double(), keys[:, g], values[:, g]
            x = torch.where(sees, q @ k.T * scale, -math.inf)
            top = torch.where(sees, (q @ k.T * scale).abs(), 0.0).amax(1)
            Q = q.abs().sum(1) * scale
            step, low = fine(ks[:, g]), fine(kl[:, g])
            mid, most = low + 8 * step, fine(k).abs().amax(1)
            if prompt:
                per_key = (d + 8) * 2 * U * (8 * step + mid.abs()) + 2.0 ** -20 * mid.abs()
                per_key = per_key + torch.where((step < 2.0 ** -8 * most.max()) & (step > 0), 2.0 ** -19 * most.max(), 0.0)
                e = Q * torch.where(sees, per_key[None], 0.0).amax(1) + d * 2.0 ** -31 * q.abs().amax(1) * most.max() * scale
            else:
                e = Q * torch.where(sees, ((d + 8) * 2 * U * (15 * step + low.abs()))[None], 0.0).amax(1)
            total = torch.logsumexp(x, 1)
            p = torch.where(sees, torch.exp(x - torch.where(total == -math.inf, 0.0, total)[:, None]), 0.0)
            v0 = torch.where(sees.any(0)[:, None], fine(v), 0.0)
            o = p @ v0
            o[(sees & ~v.isfinite().all(1)[None]).any(1)] = math.nan
            vm = torch.where(sees.any(0)[:, None], fine(vl[:, g] + 8 * vs[:, g])[:, None], 0.0)
            w = 2 * (e + 8 * U * top) + 16 * U + cnt * 2 * U
            spread = torch.stack([(p[:, :, None] * (v0[None, :, f:f + 16] - o[:, None, f:f + 16]).abs()).sum(1) for f in range(0, d, 16)], 1).flatten(1)
            t = spread * w[:, None] + 2 * U * (cnt + 8)[:, None] * (p @ ((v0 - vm).abs() + vm.abs())) + 2.0 ** -8 * o.abs() * (1 + 2.0 ** -7) + 1e-30
            if prompt:
                big = v0.abs().max()
                t = t + 2.0 ** -11 * (p @ v0.abs()) + cnt[:, None] * 2.0 ** -25 * big + p @ torch.maximum(2.0 ** -11 * v0.abs(), 2.0 ** -16 * big)
            else:
                t = t + 2.0 ** -8 * (p @ (v0 - vm).abs())
            out[row:row + T, h], tol[row:row + T, h] = o, t
            lse[row:row + T, h] = total
            lse_tol[row:row + T, h] = e + 8 * U * top + 8 * U + cnt * 2 * U + 2 * U * total.abs().nan_to_num(posinf=0.0)
    return out, tol, lse, lse_tol


def angles(n, rot, seed=0):
    """cos and sin [n][rot / 2] fp32 of a usual ladder of frequencies."""
    a = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return a.cos().float().cuda(), a.sin().float().cuda()


def rotate(x, cos, sin, position, neighbours):
    """The rotation with every product and sum rounded to fp32 and the result to x's type: what is expected bit for bit."""
    rot = 2 * cos.shape[1]
    c, s = cos[position][:, None], sin[position][:, None]
    y = x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if neighbours else (y[..., :rot // 2], y[..., rot // 2:rot])
    ac, bs, bc, as_ = a * c, b * s, b * c, a * s
    p, r = ac - bs, bc + as_
    turned = torch.stack([p, r], -1).flatten(-2) if neighbours else torch.cat([p, r], -1)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def page_scores(q, bounds, table, pages):
    """fp64 [Hkv][pages] of one sequence: q [H][d], bounds [pool][Hkv][2][d]."""
    Hkv = bounds.shape[1]
    b = bounds[table[:pages].long()].double()                       # [pages][Hkv][2][d]
    qs = q.double().view(Hkv, -1, 1, q.shape[-1])                   # [Hkv][G][1][d]
    lo, hi = b[:, :, 0].transpose(0, 1)[:, None], b[:, :, 1].transpose(0, 1)[:, None]
    return torch.maximum(qs * lo, qs * hi).sum(-1).amax(1)


def choose(scores, n_picks, page, n_sink):
    """Columns, ascending, of one sequence and KV head: the last page, those of the first slots, the largest scores (NaN the largest), the first of
    equal ones."""
    n = len(scores)
    if n <= n_picks:
        return list(range(n))
    forced = sorted(set(range(min(-(-n_sink // page), n - 1))) | {n - 1})
    s = scores.tolist()
    rest = sorted((i for i in range(n) if i not in forced), key=lambda i: (0 if math.isnan(s[i]) else 1, 0.0 if math.isnan(s[i]) else -s[i], i))
    return sorted(forced + rest[:n_picks - len(forced)])
