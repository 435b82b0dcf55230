"""Softmax attention over a paged cache on the GPU, against its definition in 64 bits."""
import math

import pytest
import torch

from paper_2607_24788_b200 import glide
from tests.paged_util import BF16, F32, Cache, check, reference

pytestmark = pytest.mark.gpu

SHAPES = [(F32, 64, 4, 4, 16), (F32, 128, 8, 4, 64), (F32, 64, 8, 1, 32), (F32, 128, 4, 1, 128), (BF16, 128, 32, 8, 64), (BF16, 64, 6, 6, 16),
          (BF16, 128, 4, 2, 256), (BF16, 64, 8, 1, 128), (BF16, 128, 8, 1, 16), (BF16, 64, 4, 1, 32), (BF16, 128, 3, 3, 32)]
MASKS = [(-1, 0), (0, 0), (0, 3), (1, 0), (16, 0), (40, 4), (7, 20), (100, 1), (1 << 40, 0)]


def decode(c, window=-1, n_sink=0, track=False, layer=0, out=None, lse=None, **kw):
    out = torch.full_like(c.q, 7.0) if out is None else out
    lse = torch.full(c.q.shape[:2], 7.0, device="cuda") if lse is None else lse
    track = dict(weight=c.weight, pos=c.pos) if track else {}
    c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, c.k, c.v, out, lse=lse, window=window, n_sink=n_sink, layer=layer, **track, **kw)
    return out, lse


def check_decode(c, window=-1, n_sink=0, track=False, layer=0):
    weight, pos = c.weight.clone(), c.pos.clone()
    out, lse = decode(c, window, n_sink, track, layer)
    want, tol, want_lse, lse_tol, given, given_tol = reference(c, window, n_sink, layer)
    check(out, want, tol, "out")
    check(lse, want_lse, lse_tol, "lse")
    c.check_pages(layer)
    if track:
        new = torch.tensor(c.lens, device="cuda") - 1
        for b in range(len(c.lens)):
            if c.lens[b]:
                weight[b, :, new[b]] = 0.0
                pos[b, :, new[b]] = new[b].int()
        check(c.weight, weight.double() + given, given_tol + given.gt(0) * weight * 2.0 ** -23, "weight")
        assert torch.equal(c.weight[given == 0], weight[given == 0]) and torch.equal(c.pos, pos)
    assert c.handle.glide_paged_device_status() == 0
    return out


@pytest.mark.parametrize("dtype,d,H,Hkv,page", SHAPES)
@pytest.mark.parametrize("window,n_sink", MASKS)
def test_decode(dtype, d, H, Hkv, page, window, n_sink):
    lens = [1, 2, 15, 16, 17, 33, 64, 100, 129, 300]
    check_decode(Cache([n - 1 for n in lens], [1] * len(lens), H, Hkv, d, dtype, page), window, n_sink, track=page != 64)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_decode_long_and_ragged(dtype):
    check_decode(Cache([20000, 0, 4095, 7, 1000], [1] * 5, 8, 2, 128, dtype, 64), track=True)
    check_decode(Cache([20000], [1], 4, 4, 64, dtype, 16), track=True)
    check_decode(Cache([9000, 5000], [1] * 2, 16, 2, 64, dtype, 32), 3000, 70, track=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_decode_of_an_empty_sequence(dtype):
    """Length 0: nothing is stored, the row is 0, its account and positions stay."""
    c = Cache([0, 49, 0], [0, 1, 0], 4, 2, 128, dtype, 16)
    c.q, c.k, c.v = (torch.cat([x * math.nan, x, x * math.nan]) for x in (c.q, c.k, c.v))
    weight, pos = c.weight.clone(), c.pos.clone()
    out, lse = decode(c, track=True)
    assert not out[0].any() and not out[2].any() and (lse[0] == -math.inf).all() and (lse[2] == -math.inf).all()
    assert out[1].isfinite().all()
    assert torch.equal(c.weight[[0, 2]], weight[[0, 2]]) and torch.equal(c.pos[[0, 2]], pos[[0, 2]])


def test_decode_many_sequences():
    """More sequences than SMs, most of them short, one long."""
    lens = [(37 * i) % 90 + 1 for i in range(400)]
    lens[123] = 5000
    check_decode(Cache([n - 1 for n in lens], [1] * 400, 4, 1, 64, BF16, 16), track=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_decode_without_new_rows_and_seen(dtype):
    """k, v None: the token is in the cache already and its account is kept; seen says the positions."""
    c = Cache([99, 10], [1, 1], 4, 2, 64, dtype, 32)
    seen = torch.tensor([500, 11], dtype=torch.int32, device="cuda")
    first, _ = decode(c, track=True, seen=seen)
    assert (c.pos[0, :, 99] == 499).all() and (c.pos[1, :, 10] == 10).all()
    weight = c.weight.clone()
    again = torch.empty_like(first)
    c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, None, None, again, weight=c.weight)
    given, given_tol = reference(c)[4:]
    assert torch.equal(first, again)
    check(c.weight, weight.double() + given, given_tol + weight * 2.0 ** -23, "weight")
    c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, None, None, again, weight=c.weight, window=0)   # sees nothing, keeps the account
    assert not again.any()
    check(c.weight, weight.double() + given, given_tol + weight * 2.0 ** -23, "weight")


def run_prefill(c, window=-1, n_sink=0, layer=0, track=False):
    out = torch.full_like(c.q, 7.0)
    lse = torch.full(c.q.shape[:2], 7.0, device="cuda")
    kw = dict(weight=c.weight, pos=c.pos) if track else {}
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, out, lse=lse, window=window, n_sink=n_sink, layer=layer, **kw)
    return out, lse


def check_prefill(c, window=-1, n_sink=0, layer=0, weights=True):
    weight, pos = c.weight.clone(), c.pos.clone()
    out, lse = run_prefill(c, window, n_sink, layer, track=weights)
    want, tol, want_lse, lse_tol, given, given_tol = reference(c, window, n_sink, layer)
    check(out, want, tol, "out")
    check(lse, want_lse, lse_tol, "lse")
    c.check_pages(layer)
    if weights:
        for b, n in enumerate(c.lens):
            weight[b, :, c.before[b]:n] = 0.0
            pos[b, :, c.before[b]:n] = torch.arange(c.before[b], n, device="cuda", dtype=torch.int32)
        assert torch.equal(c.weight, weight) and torch.equal(c.pos, pos)
        c.handle.glide_paged_weights(c.table, c.lens_dev, c.starts, c.q, lse, c.weight, window=window, n_sink=n_sink, layer=layer)
        check(c.weight, weight.double() + given, given_tol + weight * 2.0 ** -23, "weight")
    assert c.handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("dtype,d,H,Hkv,page", SHAPES)
@pytest.mark.parametrize("window,n_sink", MASKS)
def test_prefill(dtype, d, H, Hkv, page, window, n_sink):
    check_prefill(Cache([0, 0, 5, 100, 0, 16, 1], [1, 70, 30, 17, 0, 129, 3], H, Hkv, d, dtype, page), window, n_sink)


@pytest.mark.parametrize("dtype,d,H,Hkv", [(F32, 64, 4, 4), (F32, 128, 8, 2), (BF16, 128, 8, 2), (BF16, 64, 8, 1), (BF16, 128, 2, 2)])
@pytest.mark.parametrize("window,n_sink", [(-1, 0), (300, 10), (64, 200)])
def test_prefill_long(dtype, d, H, Hkv, window, n_sink):
    check_prefill(Cache([0, 1500, 3000], [1111, 333, 20], H, Hkv, d, dtype, 64), window, n_sink)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prefill_a_few_tokens_behind_a_long_cache(dtype):
    check_prefill(Cache([9000], [5], 8, 2, 128, dtype, 64))
    check_prefill(Cache([9000], [1], 8, 1, 64, dtype, 16), 8000, 100)
    check_prefill(Cache([5000, 0, 100], [16, 0, 16], 4, 4, 128, dtype, 64), 4500, 1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_few_tokens_behind_a_long_cache_that_is_not_finite_everywhere(dtype, value):
    """Parts of the cache that some of the tokens do not see hold infinities and NaN."""
    c = Cache([5000, 4000], [9, 3], 4, 2, 128, dtype, 64)
    out, lse = run_prefill(c, 3000, 5)
    want, tol, want_lse, lse_tol, _, _ = reference(c, 3000, 5)
    check(out, want, tol, "out")
    bad = 2004   # of sequence 0: seen by its queries 5000 .. 5003
    page, off = c.place(0, torch.tensor(bad, device="cuda"))
    c.v_pages[0][page, :, off] = value
    got, got_lse = torch.empty_like(out), torch.empty_like(lse)
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, None, None, got, lse=got_lse, window=3000, n_sink=5)
    check(got[4:], want[4:], tol[4:], "out")
    assert not got[:4].isfinite().any() and torch.equal(got_lse, lse)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_no_sequence_are_left_alone(dtype):
    c = Cache([20, 0], [30, 50], 4, 2, 64, dtype, 16)
    pad = lambda x: torch.cat([x, torch.full_like(x, math.nan)])  # noqa: E731
    q, k, v = pad(c.q), pad(c.k), pad(c.v)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, q, k, v, out, lse=lse)
    want, tol, want_lse, lse_tol, given, given_tol = reference(c)
    check(out[:80], want, tol, "out")
    assert (out[80:] == 7.0).all() and (lse[80:] == 7.0).all()
    c.check_pages()
    weight = c.weight.clone()
    c.handle.glide_paged_weights(c.table, c.lens_dev, c.starts, q, lse, c.weight)
    check(c.weight, weight.double() + given, given_tol + weight * 2.0 ** -23, "weight")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window,n_sink", [(-1, 0), (20, 2)])
def test_strides_layers_and_layouts(dtype, window, n_sink):
    """Pages with the heads inside, two layers, and q, k, v as parts of one tensor."""
    for new in ([40, 7], [1, 1]):
        c = Cache([30, 100], new, 8, 2, 64, dtype, 32, layers=2, layout="nhd")
        T = sum(new)
        fused = torch.full((T, 8 + 2 + 2, 64), math.nan, dtype=dtype, device="cuda")
        parts = []
        at = 0
        for x in (c.q, c.k, c.v):
            fused[:, at:at + x.shape[1]] = x
            parts.append(fused[:, at:at + x.shape[1]])
            at += x.shape[1]
        wide = torch.full((T, 16, 64), 7.0, dtype=dtype, device="cuda")
        for layer in range(2):
            lse = torch.empty(T, 8, device="cuda")
            if max(new) > 1:
                c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, *parts, wide[:, 4:12], lse=lse, window=window, n_sink=n_sink, layer=layer)
            else:
                c.handle.glide_paged_decode(c.table, c.lens_dev, *parts, wide[:, 4:12], lse=lse, window=window, n_sink=n_sink, layer=layer)
            want, tol, want_lse, lse_tol, given, given_tol = reference(c, window, n_sink, layer)
            check(wide[:, 4:12], want, tol, "out")
            assert (wide[:, :4] == 7.0).all() and (wide[:, 12:] == 7.0).all()
            c.check_pages(layer)
            weight = c.weight.clone()
            c.handle.glide_paged_weights(c.table, c.lens_dev, c.starts, parts[0], lse, c.weight, window=window, n_sink=n_sink, layer=layer)
            check(c.weight, weight.double() + given, given_tol + weight * 2.0 ** -23, "weight")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scale(dtype):
    c = Cache([200, 3], [1, 1], 4, 2, 64, dtype, 16)
    c.handle = glide.GlidePaged(c.k_pages, c.v_pages, 4, 2, c.slots, softmax_scale=0.5)
    out, lse = decode(c)
    want, tol, want_lse, lse_tol, _, _ = reference(c, scale=0.5)
    check(out, want, tol, "out")
    check(lse, want_lse, lse_tol, "lse")
    c.handle = glide.GlidePaged(c.k_pages, c.v_pages, 4, 2, c.slots, softmax_scale=0.5, weights=False)
    out, lse = run_prefill(c)
    check(out, want, tol, "out")
    with pytest.raises(glide.GlideError):
        decode(c, track=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite_reach_who_sees_them_only(dtype, value):
    """One token's V (then K) is not finite: outputs of tokens that do not see it are what they are without it."""
    for which in ("v_pages", "k_pages"):
        c = Cache([40, 60], [100, 90], 4, 2, 128, dtype, 32)
        out, lse = run_prefill(c, 50, 3)
        want, tol, want_lse, lse_tol, _, _ = reference(c, 50, 3)
        check(out, want, tol, "out")
        bad = 77   # of sequence 0: seen by its queries 77 .. 126
        page, off = c.place(0, torch.tensor(bad, device="cuda"))
        getattr(c, which)[0][page, :, off] = value
        got, got_lse = torch.empty_like(out), torch.empty_like(lse)
        c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, None, None, got, lse=got_lse, window=50, n_sink=3)
        sees = torch.zeros(190, dtype=torch.bool)
        sees[bad - 40:bad - 40 + 50] = True
        check(got[~sees], want[~sees], tol[~sees], "out of those who do not see it")
        check(got_lse[~sees], want_lse[~sees], lse_tol[~sees], "lse")
        if which == "v_pages":
            assert not got[sees].isfinite().any() and torch.equal(got_lse, lse)
        # the last token of each sequence, as a decode step
        c.q, c.new = c.q[[99, 189]].contiguous(), [1, 1]
        got = torch.empty_like(c.q)
        for lens in ([140, 150], [77, 150]):   # (neither sees it, nor does a shorter sequence whose tile still holds it)
            n = torch.tensor(lens, dtype=torch.int32, device="cuda")
            c.handle.glide_paged_decode(c.table, n, c.q, None, None, got, window=50, n_sink=3)
            assert got.isfinite().all()
        check(got[1], want[189], tol[189], "out")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_key_or_a_query_that_is_not_finite(dtype, value):
    """... reaches every row, and the account of every slot, that it belongs to: one key at each place of a tile in turn."""
    n = 700
    c = Cache([0], [n], 2, 1, 64, dtype, 64)
    weight = torch.zeros_like(c.weight)
    for bad in range(0, 384, 13):
        k, q = c.k.clone(), c.q.clone()
        k[bad] = value          # (mixed signs of q: its scores are NaN)
        out, lse = torch.empty_like(q), torch.empty(n, 2, device="cuda")
        c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, q, k, c.v, out)
        assert out[bad:].isnan().all() and out[:bad].isfinite().all()
        c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, q, c.k, c.v, out, lse=lse)
        q[bad + 300] = math.nan
        weight.zero_()
        c.handle.glide_paged_weights(c.table, c.lens_dev, c.starts, q, lse, weight)
        assert weight[0, 0, :bad + 301].isnan().all() and weight[0, 0, bad + 301:n].isfinite().all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scores_of_minus_infinity_and_large_ones(dtype):
    """A row whose scores are all -inf is 0; scores of a few thousand, of either sign, overflow nothing."""
    c = Cache([31, 31], [1, 1], 2, 1, 64, dtype, 16)
    c.k_pages[0][c.table[0, :2].long(), :, :, 0] = -math.inf
    c.k[0, :, 0] = -math.inf
    c.q[0] = 0.0
    c.q[0, :, 0] = 1.0
    c.k_pages[0][c.table[0, :2].long(), :, :, 1:] = 0.0
    c.k[0, :, 1:] = 0.0
    c.q[1] *= 1000.0
    out, lse = decode(c)
    assert not out[0].any() and (lse[0] == -math.inf).all()
    want, tol, want_lse, lse_tol, _, _ = reference(c)
    check(out[1], want[1], tol[1], "out")
    check(lse[1], want_lse[1], lse_tol[1], "lse")
    out, lse = run_prefill(c)
    assert not out[0].any() and (lse[0] == -math.inf).all()
    check(out[1], want[1], tol[1], "out")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_bad_pages_and_lengths_are_recorded(dtype):
    c = Cache([64, 64], [1, 1], 4, 2, 64, dtype, 16)
    good = decode(c)[0]
    want, tol = reference(c)[:2]
    for bad in (-1, c.k_pages.shape[1], 1 << 30, -(1 << 31)):
        table = c.table.clone()
        table[0, 1] = bad
        out = torch.empty_like(good)
        c.handle.glide_paged_decode(table, c.lens_dev, c.q, c.k, c.v, out)
        assert c.handle.glide_paged_device_status() != 0
        assert torch.equal(out[1], good[1])
        c.handle.glide_paged_prefill(table, c.lens_dev, c.starts, c.q, c.k, c.v, out)
        assert c.handle.glide_paged_device_status() != 0
        table[0, 4] = bad   # the new token's page: nothing is stored
        c.handle.glide_paged_decode(table, c.lens_dev, c.q, c.k, c.v, out)
        c.handle.glide_paged_weights(table, c.lens_dev, c.starts, c.q, torch.zeros(2, 4, device="cuda"), c.weight)
        assert c.handle.glide_paged_device_status() != 0
    c.check_pages()
    for lens in ([-5, 65], [1 << 30, 65], [-(1 << 31), 65]):
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        table = c.table.clone()
        table[0] = -1
        c.handle.glide_paged_decode(table, n, c.q, c.k, c.v, out)
        assert c.handle.glide_paged_device_status() != 0
        check(out[1], want[1], tol[1], "out")
    for starts in ([0, -1, 2], [1, 0, 1], [0, 100, 101], [0, 2, 1]):
        s = torch.tensor(starts, dtype=torch.int32, device="cuda")
        c.handle.glide_paged_prefill(c.table, c.lens_dev, s, c.q, c.k, c.v, out)
        c.handle.glide_paged_weights(c.table, c.lens_dev, s, c.q, torch.zeros(2, 4, device="cuda"), c.weight)
        assert c.handle.glide_paged_device_status() != 0
    # a window in front of which the pages are gone (a new cache: calls with such starts have stored rows in other slots)
    c = Cache([64, 64], [1, 1], 4, 2, 64, dtype, 16)
    table = c.table.clone()
    table[:, :2] = -1
    c.handle.glide_paged_decode(table, c.lens_dev, c.q, c.k, c.v, out, window=30)
    c.handle.glide_paged_prefill(table, c.lens_dev, c.starts, c.q, None, None, good, window=30)
    assert c.handle.glide_paged_device_status() == 0
    want, tol = reference(c, 30)[:2]
    check(out, want, tol, "out")
    check(good, want, tol, "out")


# ---- eviction -------------------------------------------------------------------------------------


def evicted(c, weight, pos, lens, seen, budget, recent, n_sink):
    """The definition: which rows stand where afterwards."""
    B, Hkv, _ = weight.shape
    w, p = weight.clone(), pos.clone()
    k, v = c.k_pages.clone(), c.v_pages.clone()
    for b in range(B):
        n, kept = lens[b], min(lens[b], budget)
        for g in range(Hkv):
            ws, ps = weight[b, g].tolist(), pos[b, g].tolist()

            def key(j):
                x, at = ws[j], ps[j]
                if at < n_sink or at >= seen[b] - recent:
                    return 2, 0.0, j
                return (1, 0.0, j) if math.isnan(x) else (0, x, j)
            gone = set(sorted(range(n), key=key)[:n - kept])
            holes = [j for j in range(kept) if j in gone]
            movers = [j for j in range(kept, n) if j not in gone]
            assert len(holes) == len(movers)
            to, of = (torch.tensor(x, dtype=torch.long, device="cuda") for x in (holes, movers))
            w[b, g, to.to(w.device)], p[b, g, to.to(p.device)] = weight[b, g, of.to(w.device)], pos[b, g, of.to(p.device)]
            (pt, ot), (pf, of_) = c.place(b, to), c.place(b, of)
            for dst, src in ((k, c.k_pages), (v, c.v_pages)):
                dst[0, pt, g, ot] = src[0, pf, g, of_]
    return w, p, k, v


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num()) if a.is_floating_point() else torch.equal(a, b)


@pytest.mark.parametrize("dtype,d,page", [(F32, 64, 16), (BF16, 128, 64), (BF16, 64, 32), (F32, 128, 256)])
@pytest.mark.parametrize("budget,recent,n_sink", [(64, 16, 4), (1, 0, 0), (100, 100, 0), (299, 20, 1), (300, 5, 5), (7, 3, 4)])
@pytest.mark.parametrize("in_place", [True, False])
def test_evict(dtype, d, page, budget, recent, n_sink, in_place):
    lens = [300, 1, 64, 65, 0, 200, 299]
    c = Cache(lens, [0] * len(lens), 4, 2, d, dtype, page, slots=320)
    g = torch.Generator().manual_seed(budget)
    B = len(lens)
    weight = torch.randn((B, 2, 320), generator=g).exp().cuda()
    weight[torch.rand((B, 2, 320), generator=g).cuda() < 0.3] = 0.5     # many equal ones
    weight[0, 0, 5::17] = math.nan
    weight[0, 1, 3::19] = math.inf
    weight[2, 0, ::7] = -1.0
    weight[2, 0, 1::7] = 0.0
    weight[2, 0, 2::7] = -0.0
    seen = [2 * n + 3 for n in lens]
    pos = torch.stack([torch.stack([torch.randperm(max(seen), generator=g)[:320] for _ in range(2)]) for _ in range(B)]).int().cuda()
    pos[3] = 0                                     # nothing but protected slots
    if n_sink == 0 and recent:
        pos[3] = 1 << 20
    want = evicted(c, weight, pos, lens, seen, budget, recent, n_sink)
    lens_dev, seen_dev = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, seen))
    w_out, p_out = (weight.clone(), pos.clone()) if in_place else (torch.full_like(weight, 9.0), torch.full_like(pos, 9))
    w_in, p_in = (w_out, p_out) if in_place else (weight.clone(), pos.clone())
    new_lens = lens_dev if in_place else torch.empty_like(lens_dev)
    kept = torch.arange(320, device="cuda") < lens_dev.clamp(max=budget)[:, None, None]
    kept = kept.expand_as(weight)
    c.handle.glide_paged_evict(c.table, lens_dev, seen_dev, w_in, p_in, budget, new_lens, recent=recent, n_sink=n_sink, weight_out=w_out, pos_out=p_out)
    assert new_lens.tolist() == [min(n, budget) for n in lens]
    assert same(w_out[kept], want[0][kept]) and torch.equal(p_out[kept], want[1][kept])
    assert same(c.k_pages, want[2]) and same(c.v_pages, want[3])
    if in_place:
        assert same(w_out, want[0]) and torch.equal(p_out, want[1])
    else:
        assert (w_out[~kept] == 9.0).all() and (p_out[~kept] == 9).all() and same(w_in, weight) and torch.equal(p_in, pos)
    assert c.handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("n,budget", [(20000, 2000), (20000, 19999), (70000, 30000)])
def test_evict_long(n, budget):
    c = Cache([n, n // 3], [0, 0], 2, 2, 64, BF16, 64)
    g = torch.Generator().manual_seed(n)
    weight = torch.randint(0, 1 << 12, c.weight.shape, generator=g).float().cuda()    # equal ones everywhere
    pos = torch.stack([torch.stack([torch.randperm(c.slots, generator=g) for _ in range(2)]) for _ in range(2)]).int().cuda()
    seen = [c.slots, c.slots]
    want = evicted(c, weight.cpu(), pos.cpu(), c.lens, seen, budget, 50, 4)
    lens, seen = c.lens_dev.clone(), torch.tensor(seen, dtype=torch.int32, device="cuda")
    c.handle.glide_paged_evict(c.table, lens, seen, weight, pos, budget, lens, recent=50, n_sink=4)
    assert torch.equal(weight.cpu(), want[0]) and torch.equal(pos.cpu(), want[1])
    assert same(c.k_pages, want[2]) and same(c.v_pages, want[3])
    assert lens.tolist() == [min(x, budget) for x in c.lens]


# ---- how a program uses them ----------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("amp", [30.0, 300.0])
def test_scores_that_grow_by_hundreds_from_tile_to_tile(dtype, amp):
    """Weights against the first tile's maximum would leave the range of the numbers."""
    check_prefill(Cache([0, 300], [700, 200], 4, 2, 64, dtype, 64, amp=amp))
    check_prefill(Cache([0, 300], [700, 200], 4, 2, 128, dtype, 16, amp=amp), 300, 3)
    check_prefill(Cache([6000], [9], 4, 2, 128, dtype, 64, amp=amp))
    check_decode(Cache([6000, 300], [1, 1], 4, 2, 128, dtype, 64, amp=amp), track=True)
    # ... and without lse
    c = Cache([0, 300], [700, 200], 4, 2, 128, dtype, 64, amp=amp)
    out = torch.empty_like(c.q)
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, out)
    want, tol = reference(c)[:2]
    check(out, want, tol, "out")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_run_of_them_together(dtype):
    """A prompt, its weights, an eviction, then steps that each add a token and give one slot up: outputs against the definition
    over the rows that the cache holds, positions against a list that is kept beside it."""
    H, Hkv, d, page, T, budget, recent, n_sink = 4, 2, 64, 16, 150, 64, 16, 2
    c = Cache([0, 0], [T, T - 33], H, Hkv, d, dtype, page, slots=192)
    out, lse = run_prefill(c, track=True)
    c.handle.glide_paged_weights(c.table, c.lens_dev, c.starts, c.q, lse, c.weight)
    given, given_tol = reference(c)[4:]
    for b, n in enumerate(c.lens):
        check(c.weight[b, :, :n], given[b, :, :n], given_tol[b, :, :n], "weight")
    lens, seen = c.lens_dev.clone(), c.lens_dev.clone()
    g = torch.Generator().manual_seed(1)
    for step in range(6):
        host = lens.tolist()
        want = evicted(c, c.weight.cpu(), c.pos.cpu(), host, seen.tolist(), budget, recent, n_sink)
        c.handle.glide_paged_evict(c.table, lens, seen, c.weight, c.pos, budget, lens, recent=recent, n_sink=n_sink)
        assert same(c.k_pages, want[2]) and torch.equal(c.pos.cpu(), want[1]) and same(c.weight.cpu(), want[0])
        assert lens.tolist() == [budget, budget]
        lens += 1
        seen += 1
        # what the cache holds now is the past of the next token
        c.before, c.new, c.lens = [budget, budget], [1, 1], [budget + 1, budget + 1]
        c.starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
        slot = torch.arange(budget, device="cuda")
        c.dense = [[tuple(x[0][c.place(b, slot)[0], :, c.place(b, slot)[1]] for x in (c.k_pages, c.v_pages)) for b in range(2)]]
        c.q, c.k, c.v = ((torch.randn((2, h, d), generator=g) * a).to(dtype).cuda() for h, a in ((H, 2.0), (Hkv, 1.0), (Hkv, 1.0)))
        weight, out = c.weight.clone(), torch.empty_like(c.q)
        c.handle.glide_paged_decode(c.table, lens, c.q, c.k, c.v, out, weight=c.weight, pos=c.pos, seen=seen)
        ref, tol, _, _, given, given_tol = reference(c)
        check(out, ref, tol, "out")
        weight[:, :, budget] = 0.0
        check(c.weight, weight.double() + given, given_tol + weight * 2.0 ** -23, "weight")
        assert (c.pos[:, :, budget] == seen[:, None] - 1).all()
    assert c.handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_captured_steps_follow_the_lengths(dtype):
    """A captured step replayed with other lengths, inputs and a larger table; eager calls in between."""
    c = Cache([40, 200], [1, 1], 8, 2, 64, dtype, 16, slots=512)
    out, lse = decode(c, track=True)
    weight = c.weight.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, c.k, c.v, out, weight=c.weight)
    for n in ([41, 201], [17, 201], [2, 130]):
        c.lens_dev.copy_(torch.tensor(n, dtype=torch.int32))
        c.before, c.lens = [x - 1 for x in n], n
        c.dense = [[tuple(x[:m - 1] for x in rows) for rows, m in zip(c.dense[0], n)]]
        out.fill_(7.0)
        c.weight.copy_(weight)
        graph.replay()
        replayed, w = out.clone(), c.weight.clone()
        want, tol = reference(c)[:2]
        check(replayed, want, tol, "out")
        c.weight.copy_(weight)
        eager = decode(c, track=True)[0]
        assert torch.equal(eager, replayed) and torch.equal(w, c.weight)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_two_handles_on_two_streams(dtype):
    """Handles of their own over the same pages, at the same time, give what they give one after the other, bit for bit."""
    c = Cache([3000, 700], [1, 1], 8, 2, 128, dtype, 64)
    out = decode(c)[0]
    big = Cache([200, 900], [300, 40], 8, 2, 128, dtype, 64, seed=3)
    prompt, lse = run_prefill(big)
    handles = [glide.GlidePaged(x.k_pages, x.v_pages, 8, 2, x.slots) for x in (c, big)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[torch.empty_like(out) for _ in range(10)], [torch.empty_like(prompt) for _ in range(10)]]
    lses = [torch.empty_like(lse) for _ in range(10)]
    for i in range(10):
        handles[0].glide_paged_decode(c.table, c.lens_dev, c.q, None, None, got[0][i], stream=streams[0])
        handles[1].glide_paged_prefill(big.table, big.lens_dev, big.starts, big.q, None, None, got[1][i], lse=lses[i], stream=streams[1])
    torch.cuda.synchronize()
    assert all(torch.equal(x, out) for x in got[0]) and all(torch.equal(x, prompt) for x in got[1]) and all(torch.equal(x, lse) for x in lses)


def test_calls_back_to_back():
    """Steps behind one another without a wait, each with rows that the next one reads, bit for bit what they are with waits."""
    results = []
    for wait in (True, False):
        c = Cache([500, 30, 0], [1] * 3, 8, 2, 128, BF16, 64, slots=640)
        c.table[0, :10] = torch.arange(10)
        c.table[1], c.table[2] = 10, 11   # (short sequences: one page each)
        torch.cuda.synchronize()
        outs = []
        for i in range(12):
            out = torch.empty_like(c.q)
            c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, c.k, c.v, out, weight=c.weight, pos=c.pos, window=300, n_sink=4)
            if wait:
                torch.cuda.synchronize()
            c.lens_dev += 1
            outs.append(out)
        results.append((torch.stack(outs), c.weight.clone(), c.k_pages.clone()))
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.int16 if a.dtype is BF16 else torch.int32), b.view(torch.int16 if b.dtype is BF16 else torch.int32))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_most_sequences(dtype):
    """1024 of them: prompts of no, one or a few tokens behind some, then a step, their account, an eviction."""
    new = [(7 * i) % 5 for i in range(1024)]
    check_prefill(Cache([(13 * i) % 40 for i in range(1024)], new, 2, 1, 64, dtype, 16, weights=True), 20, 1)
    c = Cache([(29 * i) % 70 for i in range(1024)], [1] * 1024, 2, 1, 64, dtype, 16)
    check_decode(c, track=True)
    want = evicted(c, c.weight.cpu(), c.pos.cpu(), c.lens, c.lens, 30, 10, 2)
    lens = c.lens_dev.clone()
    c.handle.glide_paged_evict(c.table, lens, c.lens_dev, c.weight, c.pos, 30, lens, recent=10, n_sink=2)
    assert same(c.weight.cpu(), want[0]) and torch.equal(c.pos.cpu(), want[1]) and same(c.k_pages, want[2]) and same(c.v_pages, want[3])
    assert lens.tolist() == [min(n, 30) for n in c.lens] and c.handle.glide_paged_device_status() == 0


def test_evict_more_slots_than_a_block_can_hold():
    """So many units that each has one block, and more slots than its shared memory has room for."""
    n = 60000
    c = Cache([n] + [i % 50 for i in range(99)], [0] * 100, 1, 1, 64, BF16, 256)
    g = torch.Generator().manual_seed(3)
    for budget in (20000, n - 1):
        weight = torch.randint(0, 5000, c.weight.shape, generator=g).float().cuda()
        pos = torch.randint(0, 2 * n, c.weight.shape, generator=g).int().cuda()
        seen = torch.full((100,), 2 * n, dtype=torch.int32, device="cuda")
        want = evicted(c, weight.cpu(), pos.cpu(), c.lens, seen.tolist(), budget, 50, 4)
        new_lens = torch.empty_like(c.lens_dev)
        c.handle.glide_paged_evict(c.table, c.lens_dev, seen, weight, pos, budget, new_lens, recent=50, n_sink=4)
        assert torch.equal(weight.cpu(), want[0]) and torch.equal(pos.cpu(), want[1]) and same(c.k_pages, want[2]) and same(c.v_pages, want[3])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_new_tokens_and_tables_of_few_columns(dtype):
    c = Cache([30, 20], [0, 0], 4, 2, 64, dtype, 16)
    q, k = torch.zeros(5, 4, 64, dtype=dtype, device="cuda"), torch.zeros(5, 2, 64, dtype=dtype, device="cuda")
    out, lse, weight = torch.full_like(q, 7.0), torch.full((5, 4), 7.0, device="cuda"), c.weight.clone()
    for _ in range(2):
        c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, q, k, k, out, lse=lse)
        c.handle.glide_paged_weights(c.table, c.lens_dev, c.starts, q, lse, c.weight)
    assert (out == 7.0).all() and (lse == 7.0).all() and torch.equal(c.weight, weight)
    c.check_pages()
    # the handle may hold more slots than the call's table has columns for; the table's rows lie further apart
    c = Cache([40, 3], [5, 1], 4, 2, 64, dtype, 16, slots=400)
    assert c.table.shape[1] == 25
    c.table = c.table[:, :3]
    check_prefill(c, weights=False)
    assert c.handle.glide_paged_device_status() == 0
    lens = torch.tensor([49, 4], dtype=torch.int32, device="cuda")     # (a slot more than three pages hold)
    out = torch.empty(2, 4, 64, dtype=dtype, device="cuda")
    c.handle.glide_paged_decode(c.table, lens, c.q[:2].contiguous(), None, None, out)
    assert c.handle.glide_paged_device_status() == 5


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_captured_turn(dtype):
    """Prompt, account, eviction and step captured as one graph: replays with other inputs and lengths against eager calls."""
    def turn(c, t):
        c.handle.glide_paged_prefill(c.table, t["lens"], c.starts, t["q"], t["k"], t["v"], t["out"], lse=t["lse"], weight=t["weight"], pos=t["pos"], seen=t["seen"])
        c.handle.glide_paged_weights(c.table, t["lens"], c.starts, t["q"], t["lse"], t["weight"])
        c.handle.glide_paged_evict(c.table, t["lens"], t["seen"], t["weight"], t["pos"], 100, t["lens"], recent=20, n_sink=2)
        t["lens"].add_(1)
        t["seen"].add_(1)
        c.handle.glide_paged_decode(c.table, t["lens"], t["q"][:2], t["k"][:2], t["v"][:2], t["out2"], weight=t["weight"], pos=t["pos"], seen=t["seen"])

    def fresh(seed):
        c = Cache([1500, 20], [60, 90], 8, 2, 64, dtype, 32, seed=1, slots=1600)
        g = torch.Generator().manual_seed(seed)
        for name in ("q", "k", "v"):
            setattr(c, name, torch.randn(getattr(c, name).shape, generator=g).to(dtype).cuda())
        t = dict(q=c.q, k=c.k, v=c.v, out=torch.zeros_like(c.q), lse=torch.zeros(150, 8, device="cuda"), out2=torch.zeros_like(c.q[:2]),
                 weight=torch.rand(c.weight.shape, generator=g).cuda(), pos=torch.arange(c.slots, dtype=torch.int32).expand(c.pos.shape).contiguous().cuda(),
                 lens=torch.tensor([1560 - 7 * seed, 110], dtype=torch.int32, device="cuda"))
        t["seen"] = t["lens"].clone()
        return c, t

    c, t = fresh(0)
    start = {n: x.clone() for n, x in t.items()}
    pages = c.k_pages.clone(), c.v_pages.clone()

    def reset(values):
        for n, x in values.items():
            t[n].copy_(x)
        c.k_pages.copy_(pages[0])
        c.v_pages.copy_(pages[1])

    turn(c, t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    reset(start)
    with torch.cuda.graph(graph):
        turn(c, t)
    for seed in range(3):
        other, u = fresh(seed)
        reset({n: x.clone() for n, x in u.items()})
        graph.replay()
        turn(other, u)
        for n in ("out", "lse", "out2", "weight", "pos", "lens"):
            assert torch.equal(t[n], u[n]), n
        assert same(c.k_pages, other.k_pages) and same(c.v_pages, other.v_pages)
        assert c.handle.glide_paged_device_status() == 0


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 elements: pages at its end."""
    page, Hkv, d = 256, 8, 128
    n_pages = (1 << 32) // (page * Hkv * d) + 40
    pool = torch.empty((1, n_pages, Hkv, page, d), dtype=BF16, device="cuda")
    c = Cache([700, 300], [1, 20], 16, Hkv, d, BF16, page)
    far = n_pages - 1 - c.table.clamp(0, c.k_pages.shape[1] - 1)
    pool[0, n_pages - c.k_pages.shape[1]:] = c.k_pages[0].flip(0)
    low = c.handle
    out, lse = run_prefill(c)
    want, tol = reference(c)[:2]
    check(out, want, tol, "out")
    # K and V of the far pool are the same rows
    c.v_pages.copy_(c.k_pages)
    low.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, None, None, out)
    handle = glide.GlidePaged(pool, pool, 16, 2, c.slots, weights=False)
    pool[0, n_pages - c.k_pages.shape[1]:] = c.k_pages[0].flip(0)
    got = torch.empty_like(out)
    handle.glide_paged_prefill(far.int(), c.lens_dev, c.starts, c.q, None, None, got)
    assert torch.equal(got, out)
    last = c.starts[1:].long() - 1
    q = c.q[last].contiguous()
    a, b = torch.empty_like(q), torch.empty_like(q)
    low.glide_paged_decode(c.table, c.lens_dev, q, None, None, a)
    handle.glide_paged_decode(far.int(), c.lens_dev, q, None, None, b)
    assert torch.equal(a, b)


def test_refused_calls_launch_nothing():
    c = Cache([20, 20], [1, 1], 4, 2, 64, BF16, 16)
    out = torch.full_like(c.q, 7.0)
    h = c.handle

    def refused(**kw):
        args = dict(table=c.table, lens=c.lens_dev, q=c.q, k=c.k, v=c.v, out=out, weight=None, pos=None) | kw
        with pytest.raises((glide.GlideError, AssertionError)):
            h.glide_paged_decode(**args)

    refused(layer=1)
    refused(layer=-1)
    refused(n_sink=-1)
    refused(q=c.q.float())
    refused(q=c.q[:, :2])
    refused(k=None)
    refused(lens=c.lens_dev.long())
    refused(table=c.table.long())
    refused(table=c.table.T)
    refused(weight=c.weight[:, :, :8])
    refused(weight=c.weight[:, :, :4].contiguous())
    refused(table=c.table.repeat(3, 1), lens=c.lens_dev.repeat(3))
    refused(out=out.cpu())
    refused(q=torch.empty(2, 4, 128, dtype=BF16, device="cuda")[:, :, :64])
    refused(q=torch.zeros(4 * 64 * 2 + 4, dtype=BF16, device="cuda")[4:].view(2, 4, 64))   # 8 bytes off
    assert (out == 7.0).all()
    for kw in (dict(budget=0), dict(budget=10, recent=8, n_sink=3), dict(budget=10, recent=-1)):
        with pytest.raises(glide.GlideError):
            h.glide_paged_evict(c.table, c.lens_dev, c.lens_dev, c.weight, c.pos, new_lens=c.lens_dev, **kw)
    assert h.glide_paged_device_status() == 0
