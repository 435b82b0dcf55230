"""The README's examples of the paged cache's further operators: they run, and each layer comes out as its definition says."""
import os

import pytest
import torch

from paper_2607_24788_b200 import glide
from tests.paged_more_util import BF16, Cache4, angles, reference4, rotate
from tests.paged_util import Cache, check, reference

pytestmark = pytest.mark.gpu


def block(word):
    """The README's lines around the first one that holds `word`."""
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        lines = f.read().split("\n")
    first = last = next(i for i, x in enumerate(lines) if x.startswith("    ") and word in x)
    while lines[first - 1].startswith("    "):
        first -= 1
    while last < len(lines) and lines[last].startswith("    "):
        last += 1
    return "\n".join(x[4:] for x in lines[first:last])


@pytest.mark.parametrize("word", ["turn = glide", "k_codes, v_codes, n_q_heads"])
def test_example(word):
    codes = "codes" in word
    L, B, H, Hkv, d, page, T = 2, 2, 32, 4, 128, 64, [300, 190]
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)  # noqa: E731
    ids = torch.randperm(16, generator=torch.Generator().manual_seed(0)).int().cuda()
    cos, sin = angles(512, d)
    names = dict(glide=glide, L=L, cos=cos, sin=sin, table=ids.view(B, 8), lens=torch.tensor(T, dtype=torch.int32, device="cuda"),
                 starts=torch.tensor([0, T[0], sum(T)], dtype=torch.int32, device="cuda"), q=rnd(L, sum(T), H, d) * 2, k=rnd(L, sum(T), Hkv, d),
                 v=rnd(L, sum(T), Hkv, d), q1=rnd(L, B, H, d), k1=rnd(L, B, Hkv, d), v1=rnd(L, B, Hkv, d), out=torch.zeros(L, sum(T), H, d, dtype=BF16, device="cuda"),
                 o1=torch.zeros(L, B, H, d, dtype=BF16, device="cuda"))
    if codes:
        names["turn"] = glide.GlideRotation(cos, sin)
        names["k_codes"], names["v_codes"] = (torch.zeros(L, 16, Hkv, page * glide.paged4_row_bytes(d), dtype=torch.uint8, device="cuda") for _ in range(2))
    else:
        names["k_pages"], names["v_pages"] = (torch.zeros(L, 16, Hkv, page, d, dtype=BF16, device="cuda") for _ in range(2))
        names.update(bounds=torch.zeros(L, 16, Hkv, 2, d, dtype=BF16, device="cuda"), picks=torch.zeros(B, Hkv, 64, dtype=torch.int32, device="cuda"),
                     scores=torch.zeros(B, Hkv, 8, dtype=torch.float64, device="cuda"))
    given = {n: x.clone() for n, x in names.items() if torch.is_tensor(x)}
    exec(block(word), names)
    at = torch.cat([torch.arange(n) for n in T]).cuda()
    for l in range(L):
        c = object.__new__(Cache4 if codes else Cache)
        c.H, c.Hkv, c.G, c.d, c.dtype, c.weight = H, Hkv, H // Hkv, d, BF16, torch.zeros(B, Hkv, 512, device="cuda")
        refer = (lambda c, prompt: reference4(c, prompt=prompt)) if codes else (lambda c, prompt: reference(c))  # noqa: E731
        empty = torch.zeros(0, Hkv, d, dtype=BF16, device="cuda")
        c.before, c.new, c.lens, c.starts, c.dense = [0, 0], T, T, given["starts"], [[(empty, empty)] * B]
        c.q, c.k, c.v = rotate(given["q"][l], cos, sin, at, False), rotate(given["k"][l], cos, sin, at, False), given["v"][l]
        check(names["out"][l], *refer(c, True)[:2], f"out {l}")
        c.dense = [[c.rows(0, b) for b in range(B)]]
        c.before, c.new, c.lens, c.starts = T, [1, 1], [n + 1 for n in T], torch.arange(B + 1, dtype=torch.int32, device="cuda")
        last = torch.tensor(T, device="cuda")
        c.q, c.k, c.v = rotate(given["q1"][l], cos, sin, last, False), rotate(given["k1"][l], cos, sin, last, False), given["v1"][l]
        check(names["o1"][l], *refer(c, False)[:2], f"o1 {l}")
