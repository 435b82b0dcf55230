"""Tokens on their way into a paged cache: rotation, storing, reading back, the pages' bounds."""
import math

import pytest
import torch

from paper_2607_24788_b200 import glide
from tests.paged_more_util import BF16, Cache4, angles, rotate
from tests.paged_util import F32, Cache

pytestmark = pytest.mark.gpu


def positions(c, seen):
    return torch.cat([torch.arange(s - t, s) for s, t in zip(seen, c.new)]).cuda()


@pytest.mark.parametrize("dtype,d,H,Hkv,page", [(F32, 64, 4, 4, 16), (F32, 128, 8, 1, 64), (BF16, 128, 32, 8, 64), (BF16, 64, 6, 6, 16), (BF16, 128, 4, 2, 256)])
@pytest.mark.parametrize("part,neighbours", [(1, False), (1, True), (2, False), (2, True), (0, False)])
def test_append(dtype, d, H, Hkv, page, part, neighbours):
    """Rows, queries, account and positions, bit for bit (part 0: no rotation); nothing else in the pool changes."""
    c = Cache([0, 3, 100, 0, 15], [1, 70, 30, 0, 17], H, Hkv, d, dtype, page, layers=2)
    seen = [1, 73, 1130, 5, 40]
    rotation = None
    k, q = c.k, c.q
    if part:
        cos, sin = angles(1200, d // part)
        rotation = glide.GlideRotation(cos, sin, neighbours)
        k, q = (rotate(x, cos, sin, positions(c, seen), neighbours) for x in (c.k, c.q))
    weight, pos = c.weight.clone(), c.pos.clone()
    out = torch.full_like(c.q, 7.0)
    given = c.q.clone(), c.k.clone(), c.v.clone()
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, out, rotation=rotation, weight=c.weight, pos=c.pos,
                                seen=torch.tensor(seen, dtype=torch.int32, device="cuda"), layer=1)
    assert torch.equal(out, q) and all(torch.equal(a, b) for a, b in zip(given, (c.q, c.k, c.v)))
    got_k, got_v = torch.full_like(c.k, 7.0), torch.full_like(c.v, 7.0)
    c.handle.glide_paged_read(c.table, c.lens_dev, c.starts, got_k, got_v, layer=1)
    assert torch.equal(got_k, k) and torch.equal(got_v, c.v)
    c.k = k
    c.check_pages(1)
    c.check_pages(0, stored=False)
    for b, n in enumerate(c.lens):
        weight[b, :, c.before[b]:n] = 0.0
        pos[b, :, c.before[b]:n] = torch.arange(seen[b] - c.new[b], seen[b], device="cuda", dtype=torch.int32)
    assert torch.equal(c.weight, weight) and torch.equal(c.pos, pos)
    # in place
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, c.q, given[1], c.v, c.q, rotation=rotation, seen=torch.tensor(seen, dtype=torch.int32, device="cuda"), layer=1)
    assert torch.equal(c.q, q)
    c.check_pages(1)
    assert c.handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_steps_tokens(dtype):
    """starts None: one for each sequence, none for an empty one; more sequences than a warp looks at at once."""
    B = 70
    c = Cache([(i * 13) % 50 for i in range(B)], [1] * B, 4, 2, 64, dtype, 16)
    lens = c.lens_dev.clone()
    lens[5] = 0
    cos, sin = angles(64, 64)
    out = torch.full_like(c.q, 7.0)
    c.handle.glide_paged_append(c.table, lens, None, c.q, c.k, c.v, out, rotation=glide.GlideRotation(cos, sin))
    pos = torch.tensor(c.lens, device="cuda") - 1
    want = rotate(c.q, cos, sin, pos, False)
    want[5] = 7.0
    assert torch.equal(out, want)
    c.k = rotate(c.k, cos, sin, pos, False)
    k, v = torch.empty_like(c.k), torch.empty_like(c.v)
    c.handle.glide_paged_read(c.table, lens, None, k, v)
    keep = torch.arange(B) != 5
    assert torch.equal(k[keep], c.k[keep]) and torch.equal(v[keep], c.v[keep])
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    again = torch.full_like(c.q, 7.0)
    c.handle.glide_paged_append(c.table, c.lens_dev, starts, c.q, c.k, c.v, again, rotation=glide.GlideRotation(cos, sin))
    assert torch.equal(again[keep], want[keep])
    assert c.handle.glide_paged_device_status() == 0


def test_rows_of_no_sequence_and_views():
    """Rows behind the last sequence are left alone; strided tokens and tables of angles."""
    c = Cache([10, 20], [5, 9], 4, 2, 64, BF16, 16)
    wide_q, wide_k, wide_v = (torch.full((17, 6, 64), 3.0, dtype=BF16, device="cuda") for _ in range(3))
    wide_q[:14, :4], wide_k[:14, :2], wide_v[:14, :2] = c.q, c.k, c.v
    table = torch.zeros(40, 80, device="cuda")
    cos, sin = angles(40, 32)
    table[:, :16], table[:, 40:56] = cos, sin
    out = torch.full((17, 5, 64), 7.0, dtype=BF16, device="cuda")
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, wide_q[:, :4], wide_k[:, :2], wide_v[:, :2], out[:, :4],
                                rotation=glide.GlideRotation(table[:, :16], table[:, 40:56]))
    p = positions(c, c.lens)
    assert torch.equal(out[:14, :4], rotate(c.q, cos, sin, p, False)) and (out[14:] == 7.0).all() and (out[:, 4] == 7.0).all()
    c.k = rotate(c.k, cos, sin, p, False)
    c.check_pages()
    k = torch.full((17, 2, 64), 7.0, dtype=BF16, device="cuda")
    v = k.clone()
    c.handle.glide_paged_read(c.table, c.lens_dev, c.starts, k, v)
    assert torch.equal(k[:14], c.k) and (k[14:] == 7.0).all() and (v[14:] == 7.0).all()


def test_what_is_recorded():
    c = Cache([10], [3], 4, 2, 64, BF16, 16)
    cos, sin = angles(12, 64)
    out = torch.empty_like(c.q)
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, out, rotation=glide.GlideRotation(cos, sin))   # position 12
    assert c.handle.glide_paged_device_status() == 6
    c.handle.glide_paged_append(c.table, torch.full_like(c.lens_dev, 2), c.starts, c.q, c.k, c.v, out)   # more tokens than the length
    assert c.handle.glide_paged_device_status() == 5
    c.handle.glide_paged_append(torch.full_like(c.table, -1), c.lens_dev, c.starts, None, c.k, c.v)
    assert c.handle.glide_paged_device_status() == 4
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, c.q[:0], c.k[:0], c.v[:0], out[:0])   # no token: nothing is done
    assert c.handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("dtype,d,Hkv,page", [(F32, 64, 4, 16), (F32, 128, 1, 64), (BF16, 128, 8, 64), (BF16, 64, 3, 256), (BF16, 128, 11, 32)])
def test_bounds(dtype, d, Hkv, page):
    """Of the pages with new tokens, over all slots below the length; the others' are left alone."""
    c = Cache([0, 3, 100, 0, 15, 64], [1, 70, 30, 0, 17, 300], Hkv, Hkv, d, dtype, page)
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, None, c.k, c.v)
    pages = c.k_pages.shape[1]
    for from_start in (False, True):
        bounds = torch.full((pages, Hkv, 2, d), 7.0, dtype=dtype, device="cuda")
        want = bounds.clone()
        before = [0] * 6 if from_start else c.before
        new = [n - a for n, a in zip(c.lens, before)]
        starts = torch.tensor([0] + new).cumsum(0).to(torch.int32).cuda()
        for b, (n, a) in enumerate(zip(c.lens, before)):
            for col in range(a // page, -(-n // page) if n > a else 0):
                x = c.rows(0, b)[0][col * page:min(n, (col + 1) * page)]
                want[int(c.table[b, col])] = torch.stack([x.amin(0), x.amax(0)], 1)
        c.handle.glide_paged_bounds(c.table, c.lens_dev, starts, bounds, n_tokens=sum(new) if from_start else None)
        assert torch.equal(bounds, want)
    bounds.fill_(7.0)
    c.handle.glide_paged_bounds(c.table, c.lens_dev, None, bounds)   # the newest page of each
    for b, n in enumerate(c.lens):
        if n:
            assert torch.equal(bounds[int(c.table[b, (n - 1) // page])], want[int(c.table[b, (n - 1) // page])])
    assert c.handle.glide_paged_device_status() == 0


def test_bounds_of_nan_and_infinities():
    c = Cache([0], [20], 2, 2, 64, BF16, 16)
    c.k[3, 0, 5], c.k[4, 1, 6], c.k[18, 0, 7] = math.nan, math.inf, -math.inf
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, None, c.k, c.v)
    bounds = torch.zeros((c.k_pages.shape[1], 2, 2, 64), dtype=BF16, device="cuda")
    c.handle.glide_paged_bounds(c.table, c.lens_dev, c.starts, bounds)
    a, b = bounds[int(c.table[0, 0])], bounds[int(c.table[0, 1])]
    assert a[0, :, 5].isnan().all() and a[1, 1, 6] == math.inf and b[0, 0, 7] == -math.inf
    assert int(bounds.isnan().sum()) == 2 and int(bounds.isinf().sum()) == 2


def test_captured_on_another_stream():
    c = Cache4([100, 30], [1, 1], 4, 2, 128, 16, stored=False)
    cos, sin = angles(256, 128)
    turn = glide.GlideRotation(cos, sin)
    lens, out = c.lens_dev.clone(), torch.empty_like(c.q)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.handle.glide_paged_append(c.table, lens, None, c.q, c.k, c.v, out, rotation=turn)
    graph.replay()
    pos = torch.tensor(c.lens, device="cuda") - 1
    assert torch.equal(out, rotate(c.q, cos, sin, pos, False))
    c.k = rotate(c.k, cos, sin, pos, False)
    c.check_pages()
    assert c.handle.glide_paged_device_status() == 0
