"""Calls of the paged attention that its documentation allows, beside the ordinary ones: tokens that are in the cache already, tables
whose unseen entries hold anything, no tokens at all."""
import math
import os

import pytest
import torch

from paper_2607_24788_b200 import glide
from tests.paged_util import BF16, F32, Cache, check, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_account_and_positions_of_a_prompt_that_is_in_the_cache(dtype):
    """k, v None: the new slots' account starts at 0 and their positions are written all the same, also where nothing is seen and the
    table holds nothing."""
    c = Cache([0, 40, 5], [30, 17, 0], 4, 2, 64, dtype, 16)
    out = torch.empty_like(c.q)
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, out)
    start, want_weight, want_pos = (c.weight.clone(), c.pos.clone()), c.weight.clone(), c.pos.clone()
    seen = torch.tensor([30, 1057, 9], dtype=torch.int32, device="cuda")
    for b, first in ((0, 0), (1, 1040)):
        new = slice(c.before[b], c.lens[b])
        want_weight[b, :, new] = 0.0
        want_pos[b, :, new] = torch.arange(first, first + c.new[b], dtype=torch.int32, device="cuda")
    for window, table in ((-1, c.table), (0, torch.full_like(c.table, -1))):
        c.weight.copy_(start[0])
        c.pos.copy_(start[1])
        c.handle.glide_paged_prefill(table, c.lens_dev, c.starts, c.q, None, None, out, window=window, weight=c.weight, pos=c.pos, seen=seen)
        assert torch.equal(c.weight, want_weight) and torch.equal(c.pos, want_pos)
        check(out, *reference(c, window)[:2], "out")
    c.check_pages()
    assert c.handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_position_of_a_step_that_is_in_the_cache(dtype):
    """k, v None: the slot's position is written, its account goes on from what it is."""
    c = Cache([99, 10, 0], [1, 1, 1], 4, 2, 64, dtype, 16)
    out, again = torch.empty_like(c.q), torch.empty_like(c.q)
    c.handle.glide_paged_decode(c.table, c.lens_dev, c.q, c.k, c.v, out)
    weight, pos = c.weight.clone(), c.pos.clone()
    seen = torch.tensor([500, 11, 7], dtype=torch.int32, device="cuda")
    for window, table in ((-1, c.table), (0, torch.full_like(c.table, -1))):
        for track in (dict(weight=c.weight, pos=c.pos), dict(pos=c.pos)):
            c.weight.copy_(weight)
            c.pos.copy_(pos)
            c.handle.glide_paged_decode(table, c.lens_dev, c.q, None, None, again, window=window, seen=seen, **track)
            want, tol, _, _, given, given_tol = reference(c, window)
            check(again, want, tol, "out")
            if "weight" not in track:
                given.zero_()
            check(c.weight, weight.double() + given, given_tol + weight * 2.0 ** -23, "weight")
            want_pos = pos.clone()
            for b, n in enumerate(c.lens):
                want_pos[b, :, n - 1] = seen[b] - 1
            assert torch.equal(c.pos, want_pos)
    assert c.handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window,n_sink", [(20, 2), (0, 3), (40, 0)])
def test_table_entries_that_nobody_sees_may_hold_anything(dtype, window, n_sink):
    """So many units that the fp32 account takes 64 slots at a time, which span four pages."""
    before = [200 + 17 * b for b in range(8)]
    for new in ([5] * 8, [1] * 8):
        c = Cache(before, new, 8, 4, 64, dtype, 16)
        lse = torch.empty(c.q.shape[:2], device="cuda")
        out = torch.empty_like(c.q)
        c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, None)
        want, tol, want_lse, lse_tol, given, given_tol = reference(c, window, n_sink)
        table, weight = c.table.clone(), c.weight.clone()
        for b, n in enumerate(c.lens):
            i, j = torch.arange(c.before[b], n)[:, None], torch.arange(n)[None]
            seen = ((j <= i) & ((j > i - window) | (j < n_sink))).any(0)
            for col in range(table.shape[1]):
                if not seen[col * 16:col * 16 + 16].any():
                    table[b, col] = (-1, 1 << 30, c.k_pages.shape[1])[col % 3]
        assert c.handle.glide_paged_device_status() == 0
        c.handle.glide_paged_prefill(table, c.lens_dev, c.starts, c.q, None, None, out, lse=lse, window=window, n_sink=n_sink)
        check(out, want, tol, "out")
        check(lse, want_lse, lse_tol, "lse")
        assert c.handle.glide_paged_device_status() == 0
        c.handle.glide_paged_weights(table, c.lens_dev, c.starts, c.q, lse, c.weight, window=window, n_sink=n_sink)
        check(c.weight, weight.double() + given, given_tol + weight * 2.0 ** -23, "weight")
        assert c.handle.glide_paged_device_status() == 0
        if max(new) == 1:
            c.handle.glide_paged_decode(table, c.lens_dev, c.q, None, None, out, window=window, n_sink=n_sink)
            check(out, want, tol, "out")
            assert c.handle.glide_paged_device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_calls_without_a_token(dtype):
    """Tensors of no rows, as a batch of sequences that wait has them."""
    c = Cache([30, 20], [0, 0], 4, 2, 64, dtype, 16)
    q, k, lse, weight = c.q[:0], c.k[:0], torch.empty(0, 4, device="cuda"), c.weight.clone()
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, q, k, k, torch.empty_like(q), lse=lse, weight=c.weight, pos=c.pos)
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, None, k, k)
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, q, None, None, torch.empty_like(q))
    c.handle.glide_paged_weights(c.table, c.lens_dev, c.starts, q, lse, c.weight)
    assert torch.equal(c.weight, weight) and c.handle.glide_paged_device_status() == 0
    c.check_pages()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,page,before", [(128, 64, [3000, 50]), (64, 16, [100, 3000])])
def test_rows_that_all_see_a_value_that_is_not_finite(dtype, d, page, before):
    """Every row is computed once more by itself, whole and in parts: its other columns are what they should be."""
    for new in ([150, 40], [6, 5]):
        c = Cache(before, new, 8, 2, d, dtype, page)
        want, tol, want_lse, lse_tol, _, _ = reference(c)
        out, lse = torch.empty_like(c.q), torch.empty(c.q.shape[:2], device="cuda")
        for b in range(2):
            page_of, off = c.place(b, torch.tensor(5, device="cuda"))
            c.v_pages[0][page_of, :, off, 3] = (math.nan, math.inf)[b]
        for i in range(2):
            c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, out, lse=lse if i else None)
            assert not out[..., 3].isfinite().any()
            some = [x for x in range(d) if x != 3]
            check(out[..., some], want[..., some], tol[..., some], "out")
        check(lse, want_lse, lse_tol, "lse")
        assert c.handle.glide_paged_device_status() == 0


def test_one_handle_from_two_threads():
    """Calls of several launches, issued by two threads on one stream: bit for bit what they give one after the other."""
    import threading
    c = Cache([3000, 700], [6, 6], 8, 2, 64, BF16, 64)
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, None, c.k, c.v)
    stream = torch.cuda.current_stream()
    q = [[torch.randn_like(c.q) for _ in range(2)] for _ in range(2)]
    want, got = [[], []], [[], []]

    def calls(i, results, n):
        for k in range(n):
            out, lse, weight = torch.empty_like(c.q), torch.empty(12, 8, device="cuda"), torch.zeros_like(c.weight)
            kw = dict(window=(-1, 900)[i], stream=stream)
            c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, q[i][k % 2], None, None, out, lse=lse, **kw)   # (parts and join)
            c.handle.glide_paged_decode(c.table, c.lens_dev, q[i][k % 2][:2], None, None, out[:2], weight=weight, **kw)   # (step and account)
            results[i].append((out, lse, weight))

    for i in range(2):
        calls(i, want, 2)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=calls, args=(i, got, 100)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(2):
        assert len(got[i]) == 100
        for k, x in enumerate(got[i]):
            assert all(torch.equal(a, b) for a, b in zip(x, want[i][k % 2]))
    assert c.handle.glide_paged_device_status() == 0


def readme_example():
    """The README's lines that use GlidePaged."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "README.md")) as f:
        lines = f.read().split("\n")
    first = next(i for i, x in enumerate(lines) if "GlidePaged(" in x)
    while lines[first - 1].startswith("    "):
        first -= 1
    last = first
    while last < len(lines) and lines[last].startswith("    "):
        last += 1
    return "\n".join(x[4:] for x in lines[first:last])


def test_the_readme_example():
    """Layers that share a table and lengths: each comes out as it does by itself."""
    L, B, H, Hkv, d, page, T = 2, 2, 32, 4, 64, 64, [4200, 4300]
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)  # noqa: E731
    slots = 4352
    ids = torch.randperm(B * slots // page, generator=torch.Generator().manual_seed(0)).int().cuda()
    start = dict(k_pages=torch.zeros(L, len(ids), Hkv, page, d, dtype=BF16, device="cuda"), w=torch.rand(L, B, Hkv, slots, device="cuda"),
                 v_pages=torch.zeros(L, len(ids), Hkv, page, d, dtype=BF16, device="cuda"), pos=torch.zeros(L, B, Hkv, slots, dtype=torch.int32, device="cuda"),
                 q=rnd(L, sum(T), H, d) * 3, k=rnd(L, sum(T), Hkv, d), v=rnd(L, sum(T), Hkv, d), q1=rnd(L, B, H, d), k1=rnd(L, B, Hkv, d), v1=rnd(L, B, Hkv, d),
                 out=torch.zeros(L, sum(T), H, d, dtype=BF16, device="cuda"), o1=torch.zeros(L, B, H, d, dtype=BF16, device="cuda"),
                 lse=torch.zeros(sum(T), H, device="cuda"), table=ids.view(B, -1), lens=torch.tensor(T, dtype=torch.int32, device="cuda"),
                 new_lens=torch.zeros(B, dtype=torch.int32, device="cuda"), starts=torch.tensor([0, T[0], sum(T)], dtype=torch.int32, device="cuda"))
    start["seen"] = start["lens"].clone()
    shared = {n: x.clone() for n, x in start.items()}
    exec(readme_example(), dict(glide=glide, L=L, **shared))
    assert shared["lens"].tolist() == [4097, 4097] and shared["seen"].tolist() == [4201, 4301]
    assert (shared["w"][:, :, :, 4096] > 0).all() and (shared["pos"][..., 4096] == shared["seen"][:, None] - 1).all()
    per_layer = {"k_pages", "v_pages", "w", "pos", "q", "k", "v", "q1", "k1", "v1", "out", "o1"}
    for l in range(L):
        alone = {n: (x[l:l + 1] if n in per_layer else x).clone() for n, x in start.items()}
        exec(readme_example(), dict(glide=glide, L=1, **alone))
        for n in sorted(per_layer):
            assert torch.equal(alone[n][0], shared[n][l]), (l, n)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window,n_sink", [(-1, 0), (300, 4)])
def test_outputs_with_row_sums_and_without(dtype, window, n_sink):
    for before, new in (([100, 0, 1500], [300, 200, 5]), ([2500], [6])):
        c = Cache(before, new, 8, 2, 128, dtype, 64)
        c.q[:, ::2] *= 50.0   # (references that move)
        out = [torch.empty_like(c.q) for _ in range(2)]
        for i in range(2):
            c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, c.k, c.v, out[i], window=window, n_sink=n_sink,
                                         lse=torch.empty(c.q.shape[:2], device="cuda") if i else None)
        assert torch.equal(*out) and out[0].isfinite().all()
