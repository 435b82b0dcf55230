"""A paged cache held in 4 bits: what is stored, what is read back, and attention over it, against the definitions in 64 bits."""
import math

import pytest
import torch

from paper_2607_24788_b200 import glide
from tests.paged_more_util import BF16, Cache4, levels, reference4
from tests.paged_util import check

pytestmark = pytest.mark.gpu

SHAPES = [(128, 32, 8, 64), (64, 6, 6, 16), (128, 4, 2, 256), (64, 8, 1, 128), (128, 8, 1, 16), (64, 4, 1, 32), (128, 3, 3, 32), (64, 4, 2, 64)]
MASKS = [(-1, 0), (0, 0), (0, 3), (1, 0), (16, 0), (40, 4), (7, 20), (100, 1), (1 << 40, 0)]


def check_decode(c, window=-1, n_sink=0, layer=0, new=False):
    out, lse = torch.full_like(c.q, 7.0), torch.full(c.q.shape[:2], 7.0, device="cuda")
    k, v = (c.k, c.v) if new else (None, None)
    c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, k, v, out, lse=lse, window=window, n_sink=n_sink, layer=layer)
    want, tol, want_lse, lse_tol = reference4(c, window, n_sink, layer)
    check(out, want, tol, "out")
    check(lse, want_lse, lse_tol, "lse")
    c.check_pages(layer)
    assert c.handle.glide_paged_device_status() == 0
    return out


def check_prefill(c, window=-1, n_sink=0, layer=0, new=False, with_lse=True):
    out, lse = torch.full_like(c.q, 7.0), torch.full(c.q.shape[:2], 7.0, device="cuda")
    k, v = (c.k, c.v) if new else (None, None)
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, k, v, out, lse=lse if with_lse else None, window=window, n_sink=n_sink, layer=layer)
    want, tol, want_lse, lse_tol = reference4(c, window, n_sink, layer, prompt=True)
    check(out, want, tol, "out")
    if with_lse:
        check(lse, want_lse, lse_tol, "lse")
    c.check_pages(layer)
    assert c.handle.glide_paged_device_status() == 0
    return out


@pytest.mark.parametrize("d,H,Hkv,page", SHAPES)
def test_rows_are_stored_as_their_levels(d, H, Hkv, page):
    """By append, by prefill and by decode, byte for byte, and nothing beside them; read gives the values."""
    for how in ("append", "prefill", "decode"):
        new = [1, 70, 30, 0, 17] if how != "decode" else [1] * 5
        c = Cache4([0, 3, 100, 0, 15], new, H, Hkv, d, page, stored=False, layers=2, gap=32)
        if how == "append":
            c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, None, c.k, c.v, layer=1)
        elif how == "prefill":
            c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, None, layer=1)
        else:
            c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, c.k, c.v, torch.empty_like(c.q), layer=1)
        c.check_pages(1)
        k, v = torch.full_like(c.k, 7.0), torch.full_like(c.v, 7.0)
        c.handle.glide_paged_read(c.table, c.lens_dev, c.starts if how != "decode" else None, k, v, layer=1)
        for got, x in ((k, c.k), (v, c.v)):
            code, step, low = levels(x)
            assert torch.equal(got, (code.float() * step[..., None] + low[..., None]).to(BF16))
            assert ((got.double() - x.double()).abs() <= (0.5 + 15 / 256) * step.double()[..., None] + 2.0 ** -8 * x.double().abs().amax(-1, keepdim=True)).all()
        assert c.handle.glide_paged_device_status() == 0


def test_odd_rows():
    """Rows of one value, of zeros, with infinities and NaN, of a range beyond bf16, of the least numbers, of neighbours of a border."""
    c = Cache4([0], [12], 2, 2, 64, 16, stored=False)
    g = torch.Generator().manual_seed(3)
    for x in (c.k, c.v):
        x[0], x[1, 0], x[2, :, 5], x[3, :, 9], x[4, :, 63] = 3.0, 0.0, math.inf, -math.inf, math.nan
        x[5, :, 0], x[5, :, 1] = 3.3e38, -3.3e38
        x[6] = x[6] * 2.0 ** -130
        x[7] = torch.randint(-7, 8, (2, 64), generator=g).to(BF16).cuda() * 0.5
        x[8] = x[8].abs() + 100
        x[9, :, 1:] = -0.0
        x[10] = x[10] * 1e30
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, None, c.k, c.v)
    c.check_pages()
    k, v = torch.empty_like(c.k), torch.empty_like(c.v)
    c.handle.glide_paged_read(c.table, c.lens_dev, c.starts, k, v)
    for got, x in ((k, c.k), (v, c.v)):
        assert got[2:6].isnan().all() and not got[[0, 1, 6, 7, 8, 9, 10, 11]].isnan().any()
        assert torch.equal(got[0], x[0]) and not got[1, 0].any()
    assert c.handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("d,H,Hkv,page", SHAPES)
@pytest.mark.parametrize("window,n_sink", MASKS)
def test_decode(d, H, Hkv, page, window, n_sink):
    lens = [1, 2, 15, 16, 17, 33, 64, 100, 129, 300]
    check_decode(Cache4([n - 1 for n in lens], [1] * len(lens), H, Hkv, d, page, stored=page != 64), window, n_sink, new=page == 64)


def test_decode_long_and_ragged():
    check_decode(Cache4([20000, 0, 4095, 7, 1000], [1] * 5, 8, 2, 128, 64))
    check_decode(Cache4([20000], [1], 4, 4, 64, 16))
    check_decode(Cache4([9000, 5000], [1] * 2, 16, 2, 64, 32, amp=20.0), 3000, 70)
    lens = [(37 * i) % 90 + 1 for i in range(400)]
    lens[123] = 5000
    check_decode(Cache4([n - 1 for n in lens], [1] * 400, 4, 1, 64, 16))


def test_an_empty_sequence():
    c = Cache4([0, 49, 0], [0, 1, 0], 4, 2, 128, 16)
    c.q = torch.cat([c.q * math.nan, c.q, c.q * math.nan])
    out, lse = torch.full_like(c.q, 7.0), torch.full((3, 4), 7.0, device="cuda")
    c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, None, None, out, lse=lse)
    assert not out[[0, 2]].any() and (lse[[0, 2]] == -math.inf).all() and out[1].isfinite().all()


@pytest.mark.parametrize("d,H,Hkv,page", SHAPES)
@pytest.mark.parametrize("window,n_sink", MASKS)
def test_prefill(d, H, Hkv, page, window, n_sink):
    check_prefill(Cache4([0, 0, 5, 100, 0, 16, 1], [1, 70, 30, 17, 0, 129, 3], H, Hkv, d, page, stored=page != 64), window, n_sink, new=page == 64)


@pytest.mark.parametrize("d,H,Hkv", [(128, 8, 2), (64, 8, 1), (128, 2, 2), (64, 4, 2)])
@pytest.mark.parametrize("window,n_sink", [(-1, 0), (300, 10), (64, 200)])
def test_prefill_long(d, H, Hkv, window, n_sink):
    check_prefill(Cache4([0, 1500, 3000], [1111, 333, 20], H, Hkv, d, 64), window, n_sink, with_lse=window != 300)


def test_prefill_a_few_tokens_behind_a_long_cache():
    check_prefill(Cache4([9000], [5], 8, 2, 128, 64))
    check_prefill(Cache4([9000], [1], 8, 1, 64, 16), 8000, 100)
    check_prefill(Cache4([5000, 0, 100], [16, 0, 16], 4, 4, 128, 64), 4500, 1)


@pytest.mark.parametrize("value", [math.nan, math.inf, 3e38, -3e38])
def test_what_is_not_seen_does_not_come_through(value):
    """Rows behind the window, before it, and later tokens of the same call."""
    def rows(b, k, v):
        k, v = k.clone(), v.clone()
        k[10:50, :, 3], v[10:50, :, 3] = value, value      # behind every window, in a tile with visible first slots
        return k, v
    c = Cache4([300, 290], [1, 1], 4, 2, 128, 16, rows=rows)
    assert check_decode(c, 100, 4).isfinite().all()
    c = Cache4([300, 290], [40, 150], 4, 2, 128, 16, rows=rows)
    assert check_prefill(c, 100, 4).isfinite().all()


def test_a_row_that_sees_nan_is_nan_and_no_other():
    def rows(b, k, v):
        k, v = k.clone(), v.clone()
        k[60, 0], v[70, 1] = math.nan, math.nan
        return k, v
    c = Cache4([20], [100], 4, 2, 64, 32, rows=rows)
    out = check_prefill(c)
    assert out[:40].isfinite().all() and out[50:, 2:].isnan().all() and out[40:, :2].isnan().all()
    c = Cache4([119, 50], [1, 1], 4, 2, 64, 32, rows=lambda b, k, v: rows(b, k, v) if b == 0 else (k, v))
    out = check_decode(c)
    assert out[0].isnan().all() and out[1].isfinite().all()


@pytest.mark.parametrize("of_k,of_v", [(2.0 ** -60, 2.0 ** -60), (2.0 ** -20, 2.0 ** 60), (1.0, 2.0 ** 100), (2.0 ** 20, 1.0)])
def test_scales(of_k, of_v):
    """Caches of very small and very large numbers (the queries make up for the keys')."""
    c = Cache4([700, 0], [40, 130], 4, 2, 128, 32, rows=lambda b, k, v: ((k.double() * of_k).to(BF16), (v.double() * of_v).to(BF16)))
    c.q = (c.q.double() / of_k).to(BF16)
    check_prefill(c)
    c = Cache4([700, 5], [1, 1], 4, 2, 128, 32, rows=lambda b, k, v: ((k.double() * of_k).to(BF16), (v.double() * of_v).to(BF16)))
    c.q = (c.q.double() / of_k).to(BF16)
    check_decode(c)


def test_values_and_scores_that_grow_along_the_cache():
    """Later tiles with values hundreds of times as large, and scores that leave every reference behind."""
    def rows(b, k, v):
        f = 2.0 ** (torch.arange(len(k), device="cuda", dtype=torch.float64) // 200)[:, None, None]
        return (k.double() * f.sqrt()).to(BF16), (v.double() * f).to(BF16)
    check_prefill(Cache4([900], [700], 4, 2, 128, 64, rows=rows, amp=6.0))
    check_prefill(Cache4([900], [700], 4, 2, 64, 64, rows=rows, amp=6.0), 500, 3)
    check_decode(Cache4([1600], [1], 4, 2, 128, 64, rows=rows, amp=6.0))


@pytest.mark.parametrize("zeros", [1, 128, 300])
def test_a_cache_that_begins_with_zeros(zeros):
    """Keys and values of nothing but zeros, then small ones: no scale goes by the zeros."""
    def rows(b, k, v):
        k, v = k.clone(), (v.double() * 2.0 ** -30).to(BF16)
        k[:zeros], v[:zeros] = 0.0, 0.0
        return k, v
    check_prefill(Cache4([400, 0], [60, 450], 4, 2, 128, 64, rows=rows))
    check_prefill(Cache4([400], [60], 4, 2, 64, 16, rows=rows), 250, 2)
    check_decode(Cache4([400, zeros - 1], [1, 1], 4, 2, 128, 64, rows=rows))


@pytest.mark.parametrize("d,H,Hkv,page", [(64, 16, 4, 64), (128, 16, 4, 64), (64, 4, 4, 16), (128, 8, 1, 32)])
@pytest.mark.parametrize("before,new", [(3000, 300), (0, 900), (6000, 3)])
def test_calls_that_follow_one_another(d, H, Hkv, page, before, new):
    """Two handles' calls in turns that nothing waits between give what they give by themselves, bit for bit."""
    pairs = [Cache4([before, before // 2], [new, new], H, Hkv, d, page, seed=i) for i in range(2)]
    run = lambda c, out: c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, None, None, out)  # noqa: E731
    alone = []
    for c in pairs:
        alone.append(torch.empty_like(c.q))
        run(c, alone[-1])
        torch.cuda.synchronize()
    outs = [[torch.full_like(c.q, 7.0) for c in pairs] for _ in range(20)]
    for out in outs:
        for c, o in zip(pairs, out):
            run(c, o)
    for out in outs:
        assert all(torch.equal(o, a) for o, a in zip(out, alone))


def test_layers_and_strides():
    """A second layer of padded blocks, queries and outputs that are views."""
    c = Cache4([200, 10], [30, 60], 8, 2, 128, 32, layers=3, gap=48)
    wide = torch.full((90, 12, 128), 7.0, dtype=BF16, device="cuda")
    wide[:, :8] = c.q
    out = torch.full((90, 9, 128), 7.0, dtype=BF16, device="cuda")
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, wide[:, :8], None, None, out[:, :8], layer=2)
    want, tol, _, _ = reference4(c, layer=2, prompt=True)
    check(out[:, :8], want, tol, "out")
    assert (out[:, 8] == 7.0).all()


def test_results_repeat_and_are_replayed_with_other_lengths():
    c = Cache4([5000, 300], [1, 1], 8, 2, 128, 64)
    out = torch.empty_like(c.q)
    lens = c.lens_dev.clone()
    step = lambda: c.handle.glide_paged_decode(c.table, lens, c.q, None, None, out)  # noqa: E731
    step()
    first = out.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        out.fill_(7.0)
        graph.replay()
        assert torch.equal(out, first)
    lens.copy_(torch.tensor([3000, 1], dtype=torch.int32))
    graph.replay()
    short = Cache4([2999, 0], [1, 1], 8, 2, 128, 64)
    short.dense = [[(k[:n - 1], v[:n - 1]) for (k, v), n in zip(c.dense[0], (3000, 1))]]
    rows = [c.rows(0, b) for b in range(2)]
    short.k, short.v = (torch.stack([rows[0][i][2999], rows[1][i][0]]) for i in range(2))
    short.q = c.q
    want, tol, _, _ = reference4(short)
    check(out, want, tol, "out")
    c = Cache4([300], [500], 8, 2, 128, 64)
    first, again = check_prefill(c), check_prefill(c)
    assert torch.equal(first, again)


def test_a_bad_page_and_a_bad_length_are_recorded():
    c = Cache4([100], [1], 4, 2, 64, 16)
    out = torch.empty_like(c.q)
    table = c.table.clone()
    table[0, 2] = 1 << 29
    c.handle.glide_paged_decode(table, c.lens_dev, c.q, None, None, out)
    assert c.handle.glide_paged_device_status() == 4
    c.handle.glide_paged_prefill(table, c.lens_dev, c.starts, c.q, None, None, out)
    assert c.handle.glide_paged_device_status() == 4
    c.handle.glide_paged_read(table, torch.full_like(c.lens_dev, 1 << 20), c.starts, c.k.clone(), c.v.clone())
    assert c.handle.glide_paged_device_status() in (4, 5)
    c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, None, None, out)
    assert c.handle.glide_paged_device_status() == 0
