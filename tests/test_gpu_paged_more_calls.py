"""Calls of the paged cache's further operators that their documentation allows, beside the ordinary ones: many sequences and heads, two streams at
once, captured prompts replayed with other lengths, pages that two sequences share, caches of a few slots."""
import pytest
import torch

from paper_2607_24788_b200 import glide
from tests.paged_more_util import BF16, Cache4, angles, reference4, rotate
from tests.paged_util import F32, Cache, check, reference
from tests.test_gpu_paged_sparse import Sparse

pytestmark = pytest.mark.gpu


def test_a_thousand_sequences():
    B = 1024
    c = Cache([(i * 7) % 60 for i in range(B)], [1] * B, 2, 1, 64, BF16, 16)
    s = Sparse(c, 2, 1)
    s.step(c.k, c.v)
    s.check()
    c = Cache4([(i * 7) % 60 for i in range(B)], [1 + i % 3 for i in range(B)], 2, 1, 64, 16, stored=False)
    out = torch.empty_like(c.q)
    c.handle.glide_paged_append(c.table, c.lens_dev, c.starts, None, c.k, c.v)
    c.check_pages()
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, None, None, out)
    check(out, *reference4(c, prompt=True)[:2], "out")


@pytest.mark.parametrize("H,Hkv", [(40, 40), (35, 35), (72, 9)])
def test_many_heads(H, Hkv):
    c = Cache4([100, 17], [1, 1], H, Hkv, 64, 32, stored=False)
    cos, sin = angles(128, 64)
    q = torch.empty_like(c.q)
    c.handle.glide_paged_append(c.table, c.lens_dev, None, c.q, c.k, c.v, q, rotation=glide.GlideRotation(cos, sin))
    at = torch.tensor(c.lens, device="cuda") - 1
    c.q, c.k = rotate(c.q, cos, sin, at, False), rotate(c.k, cos, sin, at, False)
    assert torch.equal(q, c.q)
    c.check_pages()
    out = torch.empty_like(q)
    c.handle.glide_paged_decode(c.table, c.lens_dev, q, None, None, out)
    check(out, *reference4(c)[:2], "out")
    d = Cache([100, 17], [1, 1], H, Hkv, 64, F32, 16)
    s = Sparse(d, 3, 1)
    s.step(d.k, d.v)
    s.check()


def test_long_pages_and_more_picks_than_columns():
    c = Cache([3000, 255, 256], [1, 1, 1], 8, 2, 128, BF16, 256)
    for n_picks in (2, 5, 1000):
        s = Sparse(c, n_picks, 300 if n_picks > 2 else 0)
        s.step(c.k, c.v)
        s.check()


def test_a_cache_of_a_few_slots():
    c = Cache4([3, 0, 10], [2, 5, 1], 4, 2, 64, 16)
    out = torch.empty_like(c.q)
    c.handle.glide_paged_prefill(c.table, c.lens_dev, c.starts, c.q, None, None, out)
    check(out, *reference4(c, prompt=True)[:2], "out")


def test_two_streams_at_once():
    """Handles of their own on streams of their own: each gives what it gives alone."""
    made = []
    for i, d in enumerate((64, 128)):
        c4 = Cache4([3000, 500], [200, 90], 8, 2, d, 32, seed=i)
        c16 = Cache([2500, 700], [1, 1], 8, 2, d, BF16, 16, seed=i)
        s = Sparse(c16, 20, 1)
        made.append((c4, s, torch.empty_like(c4.q), torch.cuda.Stream()))

    def run(c4, s, out, stream):
        c4.handle.glide_paged_prefill(c4.table, c4.lens_dev, c4.starts, c4.q, None, None, out, stream=stream)
        s.step(s.c.k, s.c.v, stream=stream)

    alone = []
    torch.cuda.synchronize()
    for m in made:
        run(*m)
        torch.cuda.synchronize()
        alone.append((m[2].clone(), m[1].out.clone(), m[1].picks.clone()))
    for _ in range(10):
        for m in made:
            run(*m)
    torch.cuda.synchronize()
    for m, a in zip(made, alone):
        assert torch.equal(m[2], a[0]) and torch.equal(m[1].out, a[1]) and torch.equal(m[1].picks, a[2])


def test_a_captured_prompt_replayed_with_other_lengths():
    """append and prefill in 4 bits, captured with room for 60 tokens, replayed with fewer: rows behind the last sequence stay as they are."""
    c = Cache4([100, 30], [40, 20], 4, 2, 128, 32, stored=False)
    cos, sin = angles(256, 128)
    turn = glide.GlideRotation(cos, sin)
    lens, starts = c.lens_dev.clone(), c.starts.clone()
    q, out = torch.full_like(c.q, 7.0), torch.full_like(c.q, 7.0)

    def call():
        c.handle.glide_paged_append(c.table, lens, starts, c.q, c.k, c.v, q, rotation=turn)
        c.handle.glide_paged_prefill(c.table, lens, starts, q, None, None, out)

    call()
    torch.cuda.synchronize()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    out.fill_(7.0)
    graph.replay()
    assert torch.equal(out, want)
    lens.copy_(torch.tensor([140, 0], dtype=torch.int32))
    starts.copy_(torch.tensor([0, 40, 40], dtype=torch.int32))
    out.fill_(7.0)
    graph.replay()
    assert torch.equal(out[:40], want[:40]) and (out[40:] == 7.0).all()
    assert c.handle.glide_paged_device_status() == 0


def test_pages_that_two_sequences_share():
    """A common beginning in the same pages, in 4 bits and with bounds."""
    c = Cache([160, 160], [1, 1], 4, 2, 64, BF16, 16)
    c.table[1, :10] = c.table[0, :10]
    c.dense[0][1] = c.dense[0][0]
    s = Sparse(c, 6, 1)
    s.step(c.k, c.v)
    s.check()
    e = Cache4([160, 160], [30, 9], 4, 2, 64, 16, stored=False)
    e.table[1, :10] = e.table[0, :10]
    e.dense[0][1] = e.dense[0][0]
    e.put(0, 0, 160)
    out = torch.empty_like(e.q)
    e.handle.glide_paged_prefill(e.table, e.lens_dev, e.starts, e.q, e.k, e.v, out)
    check(out, *reference4(e, prompt=True)[:2], "out")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append_then_the_ordinary_calls(dtype):
    """Rotated and stored by append, then a dense step and the account, as without it."""
    c = Cache([50, 7], [1, 1], 4, 2, 64, dtype, 16)
    cos, sin = angles(64, 32)
    q, out = torch.empty_like(c.q), torch.empty_like(c.q)
    weight, pos = c.weight.clone(), c.pos.clone()
    c.handle.glide_paged_append(c.table, c.lens_dev, None, c.q, c.k, c.v, q, rotation=glide.GlideRotation(cos, sin), weight=c.weight, pos=c.pos)
    at = torch.tensor(c.lens, device="cuda") - 1
    c.q, c.k = rotate(c.q, cos, sin, at, False), rotate(c.k, cos, sin, at, False)
    c.handle.glide_paged_decode(c.table, c.lens_dev, q, None, None, out, weight=c.weight)
    want, tol, _, _, given, given_tol = reference(c)
    check(out, want, tol, "out")
    for b, n in enumerate(c.lens):
        weight[b, :, n - 1], pos[b, :, n - 1] = 0.0, n - 1
    check(c.weight, weight.double() + given, given_tol + weight * 2.0 ** -23, "weight")
    assert torch.equal(c.pos, pos)
