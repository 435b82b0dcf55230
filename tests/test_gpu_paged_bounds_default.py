"""Bounds without a count of tokens, where the table has room for more than a call may bring."""
import pytest
import torch

from paper_2607_24788_b200 import glide

pytestmark = pytest.mark.gpu


def test_a_table_with_room_for_more_than_a_call_may_bring():
    """64 sequences of up to 2^25 slots: 2^31 in all, twice what n_tokens may be."""
    B, page, d, most = 64, 256, 64, 1 << 25
    g = torch.Generator().manual_seed(0)
    k = torch.randn((1, B, 1, page, d), generator=g).cuda()
    h = glide.GlidePaged(k, k.clone(), 1, B, most, weights=False)
    table = torch.full((B, most // page), -1, dtype=torch.int32)
    table[:, 0] = torch.randperm(B, generator=g)
    n = [1 + (37 * b) % page for b in range(B)]
    lens, starts = torch.tensor(n, dtype=torch.int32), torch.tensor([0] + n).cumsum(0).to(torch.int32)
    bounds = torch.full((B, 1, 2, d), 7.0, device="cuda")
    h.glide_paged_bounds(table.cuda(), lens.cuda(), starts.cuda(), bounds)
    for b in range(B):
        x = k[0, table[b, 0], 0, :n[b]]
        assert torch.equal(bounds[table[b, 0], 0], torch.stack([x.amin(0), x.amax(0)]))
    assert h.glide_paged_device_status() == 0


@pytest.mark.parametrize("count", [None, 400000])
def test_more_pages_than_blocks(count):
    """Some 25000 pages of 16 slots, of three sequences: the blocks of a launch take pages in turns."""
    page, d, n = 16, 64, [280001, 5, 119994]
    pages = [-(-i // page) for i in n]
    g = torch.Generator().manual_seed(0)
    k = torch.randn((1, sum(pages) + 2, 2, page, d), generator=g).to(torch.bfloat16).cuda()
    ids = torch.randperm(k.shape[1], generator=g).to(torch.int32)
    table = torch.full((3, max(pages)), -1, dtype=torch.int32)
    bounds = torch.full((k.shape[1], 2, 2, d), 7.0, dtype=torch.bfloat16, device="cuda")
    want = bounds.clone()
    for b in range(3):
        mine = ids[sum(pages[:b]):sum(pages[:b + 1])]
        table[b, :pages[b]] = mine
        x = k[0, mine.long().cuda()]
        last = n[b] - (pages[b] - 1) * page
        want[mine.long().cuda()] = torch.stack([x.amin(2), x.amax(2)], 2)
        want[int(mine[-1])] = torch.stack([x[-1, :, :last].amin(1), x[-1, :, :last].amax(1)], 1)
    h = glide.GlidePaged(k, k.clone(), 2, 3, 300000, weights=False)
    starts = torch.tensor([0] + n).cumsum(0).to(torch.int32)
    h.glide_paged_bounds(table.cuda(), torch.tensor(n, dtype=torch.int32).cuda(), starts.cuda(), bounds, n_tokens=count)
    assert torch.equal(bounds, want)
    assert h.glide_paged_device_status() == 0
