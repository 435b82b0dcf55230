"""What a serving program asks of the paged cache beside plain attention, as cases that can be timed: tokens that come in with their
positions' rotation, a cache held in 4 bits, and steps that read only the pages that a cheap score selects.

  op        "append": the new tokens' queries and keys are rotated by their positions, keys and values stored in their pages, the queries
                      written out; with `bounds` the least and largest key values of the pages that got tokens are brought up to date; of a
                      4-bit cache the new rows are read back, as the values that they stand for
            "decode": one token per sequence, in the cache already, attends to a cache held in 4 bits
            "prefill": the same for several tokens per sequence, each of which attends to those up to itself
            "sparse": one new token per sequence is stored, its page's bounds take it in, and for every KV head it attends to `picks` pages:
                      its own, those of the first tokens, and of the others those whose bounds allow the largest score
  heads, kv_heads, dim, dtype, page (tokens of a page), batch
  bits      of a cached value (4: 16 levels between a row's least and largest value)
  context   tokens in the cache before the pass (of the longest sequence)
  tokens    new tokens of the pass (of the longest sequence)
  ragged    the sequences' lengths differ
  window    newest tokens that a token sees, itself among them (-1: all);  sinks: first tokens that stay visible
  rotated   features that are rotated;  neighbours: feature 2i goes with 2i + 1, not i with i + rotated / 2

With `own` false, `run` computes all this from elementary torch operations in fp32, the pages' scores in fp64."""
import math

import torch

own = False

_LLAMA = dict(heads=32, kv_heads=8, dim=128, dtype="bf16", page=64, bits=16)
_LLAMA4 = dict(_LLAMA, bits=4)
_TINY = dict(heads=4, kv_heads=4, dim=64, dtype="f32", page=16, bits=32)
_PLAIN = dict(batch=1, context=0, tokens=1, ragged=False, window=-1, sinks=0, rotated=0, neighbours=False, bounds=False, picks=0)


def _case(name, op, shape, **kw):
    return dict(_PLAIN, name=name, op=op, **shape) | kw


def listed():
    return [
        # The smallest call: the token of one fp32 layer of 4 heads.
        _case("append_tiny_f32", "append", _TINY, context=512, rotated=64),
        # A serving batch's new tokens into a 4-bit cache.
        _case("append_step_4bit_b16", "append", _LLAMA4, batch=16, context=4096, ragged=True, rotated=128),
        # One long prompt, a length that is no multiple of any tile, into pages whose bounds sparse steps will read.
        _case("append_b1_8k", "append", _LLAMA, tokens=8001, rotated=128, bounds=True),
        # Prompts of different lengths into a 4-bit cache, half of the features rotated, neighbours together.
        _case("append_4bit_b8_2k", "append", _LLAMA4, batch=8, tokens=2048, ragged=True, rotated=64, neighbours=True),
        # Interactive decode of one 32K-token sequence.
        _case("decode_b1_32k", "decode", _LLAMA4, context=32768),
        # A serving batch of different lengths, a window of 1024 tokens and four first ones.
        _case("decode_sinks_b16_16k", "decode", _LLAMA4, batch=16, context=16384, ragged=True, window=1024, sinks=4),
        # Long documents: four sequences of 128K tokens.
        _case("decode_b4_128k", "decode", _LLAMA4, batch=4, context=131072),
        # One long prompt.
        _case("prefill_b1_8k", "prefill", _LLAMA4, tokens=8001),
        # A further turn of four conversations.
        _case("prefill_turn_b4_32k", "prefill", _LLAMA4, batch=4, context=32768, tokens=1000, ragged=True),
        # A few proposed tokens are checked behind a long document.
        _case("prefill_few_b1_128k", "prefill", _LLAMA4, context=131072, tokens=8),
        # Steps that read 32 of 512 pages of each of 16 sequences of different lengths ...
        _case("sparse_b16_32k", "sparse", _LLAMA, batch=16, context=32768, ragged=True, picks=32, sinks=4),
        # ... and 64 of 2048 pages of four long ones.
        _case("sparse_b4_128k", "sparse", _LLAMA, batch=4, context=131072, picks=64, sinks=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: every operator, 1 to 8 KV heads with 1 to 8 query heads each, 1 to 16 sequences of one token to 128K,
    pages of 16 to 128 tokens, fp32 and bf16 where the cache is not held in 4 bits."""
    op = rng.choice(["append", "decode", "prefill", "sparse"])
    dtype = rng.choice(["bf16", "bf16", "f32"]) if op in ("append", "sparse") else "bf16"
    kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8])
    bits = 4 if op in ("decode", "prefill") or (op == "append" and dtype == "bf16" and rng.random() < 0.6) else 32 if dtype == "f32" else 16
    shape = dict(heads=kv_heads * group, kv_heads=kv_heads, dim=rng.choice([64, 128]), dtype=dtype, page=rng.choice([16, 32, 64, 128]), bits=bits)
    batch = _log_int(rng, 1, 16)
    c = _case("", op, shape, batch=batch, ragged=rng.random() < 0.7)
    if op in ("decode", "prefill") and rng.random() < 0.5:
        c.update(window=_log_int(rng, 1, 4096), sinks=rng.choice([0, 1, 4, 100]))
    if op == "append":
        c.update(rotated=rng.choice([c["dim"], c["dim"] // 2]), neighbours=rng.random() < 0.4, bounds=bits != 4 and rng.random() < 0.5)
        c.update(tokens=max(1, _log_int(rng, 1, 8000) // batch), context=_log_int(rng, 1, 8192 // batch) if rng.random() < 0.6 else 0)
    elif op == "decode":
        c.update(context=_log_int(rng, 1, 131072 // batch))
    elif op == "prefill":
        c.update(tokens=max(1, _log_int(rng, 2, 8000) // batch))
        if rng.random() < 0.6:
            c["context"] = _log_int(rng, 1, 32768 // batch)
    else:
        c.update(context=_log_int(rng, 1, (32768 if dtype == "f32" else 131072) // batch), sinks=rng.choice([0, 1, 4]))
        c["picks"] = _log_int(rng, 2, 128)
    del c["name"]
    return c


def _lengths(case):
    """Per sequence: tokens in the cache before the pass, new tokens."""
    before, new = [], []
    for b in range(case["batch"]):
        part = 2000 if case["ragged"] else 0
        before.append(case["context"] - (b * 617 % 1000) * case["context"] // part if part else case["context"])
        new.append(max(1, case["tokens"] - (b * 389 % 1000) * case["tokens"] // part) if part else case["tokens"])
    return before, new


def _inputs(case, seed):
    """Seeded inputs on the GPU.  Keys and values have unit variance, queries four times that, so that some tokens weigh much more
    than others.  A sequence's pages lie anywhere in the pool; the table's entries behind them are -1."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    B, H, Hkv, d, page = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["page"]
    before, new = _lengths(case)
    lens = [n + t for n, t in zip(before, new)]
    used = [-(-n // page) for n in lens]
    cols, pages = max(used) + 1, sum(used) + 8

    def normal(*shape, scale=1.0):
        x = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)
        return x if scale == 1.0 else x.mul_(scale)

    ids = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    col = torch.arange(cols, device="cuda")
    count = torch.tensor(used, device="cuda")
    first = count.cumsum(0) - count
    table = torch.where(col < count[:, None], ids[(first[:, None] + col).clamp(max=pages - 1)], -1).to(torch.int32).contiguous()
    rows = sum(new)
    s = dict(case=case, table=table, starts=torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32),
             before=torch.tensor(before, device="cuda", dtype=torch.int32), lens=torch.tensor(lens, device="cuda", dtype=torch.int32),
             most=max(lens), most_new=max(new), q=normal(rows, H, d, scale=2.0))
    s["out"] = torch.zeros_like(s["q"])
    if case["bits"] == 4:
        # of every page and KV head: the slots' features, two to a byte, the even one in the low bits, then for each slot the
        # distance of the levels and the lowest one, in bf16
        shape = (1, pages, Hkv, page * d // 2)
        for n in ("k_pages", "v_pages"):
            codes = torch.randint(0, 256, shape, generator=gen, device="cuda", dtype=torch.uint8)
            low = torch.randn((1, pages, Hkv, page), generator=gen, device="cuda").mul_(0.25).sub_(2.5)
            levels = torch.stack([low.mul(-2 / 15), low], -1).to(torch.bfloat16).view(torch.uint8).flatten(3)
            s[n] = torch.cat([codes, levels], 3)
    else:
        s.update(k_pages=normal(1, pages, Hkv, page, d), v_pages=normal(1, pages, Hkv, page, d))
    if case["op"] in ("append", "sparse"):
        s.update(k=normal(rows, Hkv, d), v=normal(rows, Hkv, d))
    if case["op"] == "append":
        angle = torch.arange(max(lens), device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(0, case["rotated"], 2, device="cuda", dtype=torch.float64) / case["rotated"])
        s.update(cos=angle.cos().float(), sin=angle.sin().float())
        if case["bits"] == 4:
            s.update(k_rows=torch.zeros_like(s["k"]), v_rows=torch.zeros_like(s["v"]))
    else:
        s["lse"] = torch.zeros(rows, H, device="cuda")
    if case["bounds"] or case["op"] == "sparse":
        s["bounds"] = torch.stack([s["k_pages"][0].amin(2), s["k_pages"][0].amax(2)], 2)   # [pages][KV heads][2][d]
    if case["op"] == "sparse":
        newest = [n - 1 for n in lens]   # of the newest pages: of the tokens that were there
        for b, n in enumerate(newest):
            if n % page:
                p = int(table[b, n // page])
                x = s["k_pages"][0, p, :, :n % page]
                s["bounds"][p, :, 0], s["bounds"][p, :, 1] = x.amin(1), x.amax(1)
        s["picks"] = torch.zeros(B, Hkv, case["picks"], dtype=torch.int32, device="cuda")
        s["scores"] = torch.zeros(B, Hkv, cols, dtype=torch.float64, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2607_24788_b200 import glide
        s["cache"] = glide.GlidePaged(s["k_pages"], s["v_pages"], case["heads"], case["batch"], s["table"].shape[1] * case["page"],
                                      weights=False, **(dict(head_dim=case["dim"]) if case["bits"] == 4 else {}))
        if case["op"] == "append":
            s["rotation"] = glide.GlideRotation(s["cos"], s["sin"], neighbours=case["neighbours"])
    return s


def _outputs(s):
    case = s["case"]
    if case["op"] in ("decode", "prefill"):
        names = ["out", "lse"]
    elif case["op"] == "sparse":
        names = ["out", "lse", "picks", "k_pages", "v_pages", "bounds"]
    else:
        names = ["out"] + (["k_rows", "v_rows"] if case["bits"] == 4 else ["k_pages", "v_pages"] + ["bounds"] * case["bounds"])
    return {n: s[n] for n in names}


# ---- the calls of the framework -------------------------------------------------------------------


def _run_own(s):
    case, cache = s["case"], s["cache"]
    if case["op"] == "append":
        cache.glide_paged_append(s["table"], s["lens"], s["starts"], s["q"], s["k"], s["v"], s["out"], rotation=s["rotation"])
        if case["bounds"]:
            cache.glide_paged_bounds(s["table"], s["lens"], s["starts"], s["bounds"])
        if case["bits"] == 4:
            cache.glide_paged_read(s["table"], s["lens"], s["starts"], s["k_rows"], s["v_rows"])
    elif case["op"] == "decode":
        cache.glide_paged_decode(s["table"], s["lens"], s["q"], None, None, s["out"], lse=s["lse"], window=case["window"], n_sink=case["sinks"])
    elif case["op"] == "prefill":
        cache.glide_paged_prefill(s["table"], s["lens"], s["starts"], s["q"], None, None, s["out"], lse=s["lse"], window=case["window"],
                                  n_sink=case["sinks"])
    else:
        cache.glide_paged_decode_sparse(s["table"], s["lens"], s["q"], s["k"], s["v"], s["out"], s["bounds"], s["picks"], s["scores"], lse=s["lse"],
                                        n_sink=case["sinks"])
    return _outputs(s)


# ---- the plain forms ------------------------------------------------------------------------------


def _place(s, seq, slot):
    """Page and offset of slots of sequences."""
    page = s["case"]["page"]
    return s["table"][seq, slot // page].long(), slot % page


def _new_slots(s):
    """Of every new token: its sequence, its number among the sequence's new tokens, its slot."""
    row = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(s["starts"][1:].contiguous(), row.to(torch.int32), right=True)
    at = row - s["starts"][seq]
    return seq, at, s["before"][seq] + at


def _rotate(s, x, slot):
    case = s["case"]
    n = case["rotated"]
    cos, sin = s["cos"][slot][:, None], s["sin"][slot][:, None]
    y = x.float()
    a, b = (y[..., 0:n:2], y[..., 1:n:2]) if case["neighbours"] else (y[..., :n // 2], y[..., n // 2:n])
    turned = [a * cos - b * sin, b * cos + a * sin]
    turned = torch.stack(turned, -1).flatten(-2) if case["neighbours"] else torch.cat(turned, -1)
    return torch.cat([turned, y[..., n:]], -1).to(x.dtype)


def _levels(x):
    """Codes of rows [.., d] on 16 levels between a row's least and largest value; the distance of the levels and the lowest one."""
    x = x.float()
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    step = ((high - low) * (1.0 / 15.0)).to(torch.bfloat16).float()
    code = torch.where(step > 0.0, ((x - low) / step).round().clamp(0.0, 15.0), 0.0)
    return code, step, low


def _append(s):
    case = s["case"]
    seq, at, slot = _new_slots(s)
    page, off = _place(s, seq, slot)
    s["out"].copy_(_rotate(s, s["q"], slot))
    k = _rotate(s, s["k"], slot)
    if case["bits"] == 4:
        size, per = case["page"] * case["dim"] // 2, case["dim"] // 2
        for name, x in (("k", k), ("v", s["v"])):
            code, step, low = _levels(x)
            c = code.to(torch.uint8)
            pages, heads = s[name + "_pages"][0], torch.arange(case["kv_heads"], device="cuda")[:, None]
            pages[page[:, None, None], heads, off[:, None, None] * per + torch.arange(per, device="cuda")] = c[..., 0::2] | c[..., 1::2] << 4
            levels = torch.cat([step, low], -1).to(torch.bfloat16).view(torch.uint8)
            pages[page[:, None, None], heads, size + off[:, None, None] * 4 + torch.arange(4, device="cuda")] = levels
            s[name + "_rows"].copy_(code * step + low)
        return
    s["k_pages"][0][page, :, off] = k
    s["v_pages"][0][page, :, off] = s["v"]
    if case["bounds"]:
        # (slots behind a sequence's end count for nothing)
        col = torch.unique(torch.stack([seq, slot // case["page"]]), dim=1)
        pages = s["table"][col[0], col[1]].long()
        there = (col[1][:, None] * case["page"] + torch.arange(case["page"], device="cuda") < s["lens"][col[0]][:, None])[:, None, :, None]
        x = s["k_pages"][0][pages]
        s["bounds"][pages, :, 0] = torch.where(there, x, math.inf).amin(2)
        s["bounds"][pages, :, 1] = torch.where(there, x, -math.inf).amax(2)


def _attend(s):
    """Outputs and logarithms of the row sums of every token over the 4-bit cache."""
    case = s["case"]
    B, H, Hkv, d, T, w, n0 = case["batch"], case["heads"], case["kv_heads"], case["dim"], s["most_new"], case["window"], case["sinks"]
    G, most = H // Hkv, s["most"]
    seq, at, _ = _new_slots(s)
    if 0 <= w and n0 + w - 1 + T < most:   # the first tokens, and those that some token's window holds
        begin = (s["before"] - w + 1).clamp(min=n0)[:, None]
        slot = torch.cat([torch.arange(n0, device="cuda").expand(B, n0), begin + torch.arange(w - 1 + T, device="cuda")], 1)
    else:
        slot = torch.arange(most, device="cuda").expand(B, most)
    there = slot < s["lens"][:, None]
    page, off = _place(s, torch.arange(B, device="cuda")[:, None], slot.clamp(max=most - 1))
    mine = s["before"][:, None] + torch.arange(T, device="cuda")                    # slot of a query
    sees = there[:, None] & (slot[:, None] <= mine[..., None])
    if w >= 0:
        sees &= (slot[:, None] > mine[..., None] - w) | (slot[:, None] < n0)
    sees = sees[:, None, None]                                                       # [B][1][1][T][n]
    q = torch.zeros(B, T, H, d, device="cuda")
    q[seq, at] = s["q"].float()
    q = (q.view(B, T, Hkv, G, d).permute(0, 2, 3, 1, 4) * d ** -0.5).reshape(B, Hkv, G * T, d)
    size, per = case["page"] * d // 2, d // 2
    step = max(1, min(Hkv, (2 << 30) // (B * G * T * slot.shape[1])))
    for h in range(0, Hkv, step):
        heads = slice(h, h + step)

        def rows(name):   # [B][heads][slots][d]
            x = s[name][0][:, heads]
            codes = x[..., :size].unflatten(-1, (case["page"], per))[page, :, off].transpose(1, 2)
            levels = x[..., size:].contiguous().view(torch.bfloat16).unflatten(-1, (case["page"], 2))[page, :, off].transpose(1, 2).float()
            return torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() * levels[..., :1] + levels[..., 1:]

        k = rows("k_pages")
        n = k.shape[1]
        x = torch.matmul(q[:, heads], k.transpose(-1, -2)).view(B, n, G, T, -1).masked_fill_(~sees, -math.inf)
        del k
        top = x.amax(-1, keepdim=True)
        p = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
        total = p.sum(-1, keepdim=True)
        lse = (top + total.log()).squeeze(-1)
        total = torch.where(total == 0.0, 1.0, total)
        o = torch.matmul(p.view(B, n, G * T, -1), rows("v_pages")).view(B, n, G, T, d) / total
        s["out"].view(-1, Hkv, G, d)[:, heads] = o.permute(0, 3, 1, 2, 4)[seq, at].to(s["out"].dtype)
        s["lse"].view(-1, Hkv, G)[:, heads] = lse.permute(0, 3, 1, 2)[seq, at]


def _sparse(s):
    case = s["case"]
    B, H, Hkv, d, P, n0 = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["page"], case["sinks"]
    G, cols = H // Hkv, s["table"].shape[1]
    batch, newest = torch.arange(B, device="cuda"), (s["lens"] - 1).long()
    page, off = _place(s, batch, newest)
    s["k_pages"][0][page, :, off] = s["k"]
    s["v_pages"][0][page, :, off] = s["v"]
    k, fresh, b = s["k"], (off == 0)[:, None, None], s["bounds"]
    b[page, :, 0] = torch.where(fresh, k, torch.minimum(k, b[page, :, 0]))
    b[page, :, 1] = torch.where(fresh, k, torch.maximum(k, b[page, :, 1]))
    # scores next to the border of what is selected have to fall on the same side everywhere: 64 bits
    bounds = b[s["table"].clamp(min=0).long()].double()                              # [B][cols][KV heads][2][d]
    q = s["q"].double().view(B, Hkv, G, d)
    score = torch.einsum("bhgd,bchd->bhgc", q.clamp(min=0.0), bounds[..., 1, :]) + torch.einsum("bhgd,bchd->bhgc", q.clamp(max=0.0), bounds[..., 0, :])
    score = score.amax(2)
    col = torch.arange(cols, device="cuda")
    used = col <= newest[:, None] // P
    score = torch.where(((col == newest[:, None] // P) | (col * P < n0))[:, None], math.inf, score)
    score = torch.where(used[:, None], score, -math.inf)
    order = score.argsort(dim=2, descending=True, stable=True)[..., :case["picks"]]
    order = torch.where(torch.gather(used[:, None].expand(B, Hkv, cols), 2, order), order, cols).sort(dim=2).values
    s["picks"].fill_(-1)[..., :order.shape[2]] = torch.where(order < cols, order, -1).to(torch.int32)
    slot = (order[..., None] * P + torch.arange(P, device="cuda")).flatten(2)        # [B][KV heads][slots]
    there = slot <= newest[:, None, None]
    slot = torch.where(there, slot, 0)
    at, o = _place(s, batch[:, None, None], slot)
    head = torch.arange(Hkv, device="cuda")[:, None]
    keys, values = (x[0][at, head, o].float() for x in (s["k_pages"], s["v_pages"]))
    x = torch.matmul(s["q"].float().view(B, Hkv, G, d) * d ** -0.5, keys.transpose(-1, -2)).masked_fill_(~there[:, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = (x - top).exp()
    total = p.sum(-1, keepdim=True)
    s["out"].copy_((torch.matmul(p, values) / total).reshape(B, H, d))
    s["lse"].copy_((top + total.log()).reshape(B, H))


def run(s):
    if own:
        return _run_own(s)
    {"append": _append, "sparse": _sparse}.get(s["case"]["op"], _attend)(s)
    return _outputs(s)


def work(case):
    """One pass.  append: the new tokens' queries, keys and values and their positions' angles read, queries and rows written (and read back
    where they are held in 4 bits; the bounds written).  decode, prefill: the visible slots, queries and outputs once, multiply-adds of the
    two products.  sparse: the bounds of all pages, the slots of the selected ones, and the new tokens' tensors."""
    H, Hkv, d, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    elem = 4 if case["dtype"] == "f32" else 2
    slot = Hkv * (d + 8 if case["bits"] == 4 else 2 * d * elem)   # K and V of a slot
    before, new = _lengths(case)
    byts = flops = 0
    for n, t in zip(before, new):
        if case["op"] == "append":
            byts += 2 * t * H * d * elem + 2 * t * Hkv * d * elem + t * slot + 4 * t * case["rotated"]
            flops += 3 * t * (H + Hkv) * case["rotated"]
            if case["bits"] == 4:
                byts += t * slot + 2 * t * Hkv * d * elem
                flops += 12 * t * Hkv * d
            if case["bounds"]:
                pages = (n + t - 1) // P - n // P + 1
                byts += pages * Hkv * 2 * d * elem
                flops += 2 * t * Hkv * d
            continue
        if case["op"] == "sparse":
            pages = (n + 1 + P - 1) // P
            seen = min(n + 1, case["picks"] * P)
            byts += pages * Hkv * 2 * d * elem + seen * slot + slot + 2 * H * d * elem + 4 * case["picks"] * Hkv
            flops += 2 * pages * H * d + 4 * H * d * seen
            continue
        w = n + t if case["window"] < 0 else case["window"]
        first = min(case["sinks"], n + t)
        old = min(n, w - 1 if w else 0)
        old += max(0, min(first, n - old))
        byts += (old + t) * slot + 2 * t * H * d * elem + 4 * t * H
        flops += 4 * H * d * sum(min(i, w) + min(first, max(0, i - w)) for i in range(n + 1, n + t + 1))
    return dict(bytes=byts, flops=flops)


# ---- the definitions, in 64 bits ------------------------------------------------------------------


def _exact_append(s):
    """Token by token of each sequence, as complex numbers; bounds have no computed value."""
    case = s["case"]
    n, half = case["rotated"], case["rotated"] // 2
    before, new = _lengths(case)
    position = torch.cat([torch.arange(a, a + t, device="cuda") for a, t in zip(before, new)])
    turn = torch.complex(s["cos"].double(), s["sin"].double())[position].unsqueeze(1)
    got = {}
    for name, x in (("out", s["q"]), ("k", s["k"])):
        x = x.double().clone()
        pair = x[..., :n].unflatten(-1, (half, 2)) if case["neighbours"] else x[..., :n].unflatten(-1, (2, half)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        x[..., :n] = z.flatten(-2) if case["neighbours"] else z.transpose(-1, -2).flatten(-2)
        got[name] = x
    k = got.pop("k")
    if case["bits"] != 4:
        return got | {"k_pages": None, "v_pages": None} | ({"bounds": None} if case["bounds"] else {})
    for name, x in (("k_rows", k.to(s["q"].dtype).double()), ("v_rows", s["v"].double())):   # (what a 16-bit cache would hold has 16 levels)
        low = x.min(-1, keepdim=True).values
        step = ((x.max(-1, keepdim=True).values - low) / 15).to(torch.bfloat16).double()
        got[name] = low + step * torch.where(step > 0, torch.round((x - low) / step.clamp(min=1e-300)), 0).clamp(0, 15)
    return got


def _exact_softmax(q, keys, values, hidden=None):
    x = q @ keys.T / math.sqrt(keys.shape[1])
    if hidden is not None:
        x = x.masked_fill(hidden, -math.inf)
    total = torch.logsumexp(x, 1)
    return torch.exp(x - torch.where(total == -math.inf, 0.0, total)[:, None]) @ values, total


def exact(case, seed):
    """The definitions, sequence by sequence and head by head.  What is only moved or compared has no such value; the pages that a
    sparse step selects do."""
    s = _inputs(case, seed)
    if case["op"] == "append":
        return _exact_append(s)
    H, Hkv, d, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    G = H // Hkv
    before, new = _lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    picks = torch.full((case["batch"], Hkv, case["picks"]), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(case["batch"]):
        n, t = before[b], new[b]
        m = n + t
        pages = s["table"][b, :-(-m // P)].long()
        i = torch.arange(n, m, device="cuda")[:, None]
        j = torch.arange(m, device="cuda")[None]
        hidden = j > i
        if case["window"] >= 0:
            hidden = hidden | ((j <= i - case["window"]) & (j >= case["sinks"]))
        for h in range(Hkv):
            group = range(h * G, h * G + G)
            if case["op"] != "sparse":
                keys, values = [], []
                for name, rows in (("k_pages", keys), ("v_pages", values)):
                    x = s[name][0, pages, h]
                    codes = x[:, :P * d // 2].reshape(-1, d // 2).to(torch.int32)
                    levels = x[:, P * d // 2:].reshape(-1, 4).contiguous().view(torch.bfloat16).double()
                    rows.append(levels[:m, 1:] + levels[:m, :1] * torch.stack([codes % 16, codes // 16], 2).flatten(1)[:m].double())
                for g in group:
                    out[at:at + t, g], lse[at:at + t, g] = _exact_softmax(s["q"][at:at + t, g].double(), keys[0], values[0], hidden)
                continue
            keys = torch.cat([s["k_pages"][0, pages, h].reshape(-1, d)[:n], s["k"][at:at + 1, h]]).double()
            values = torch.cat([s["v_pages"][0, pages, h].reshape(-1, d)[:n], s["v"][at:at + 1, h]]).double()
            low, high = s["bounds"][pages, h, 0].double(), s["bounds"][pages, h, 1].double()
            newest = keys[(m - 1) // P * P:]
            low[-1], high[-1] = newest.min(0).values, newest.max(0).values
            best = torch.stack([torch.maximum(x * low, x * high).sum(1) for x in s["q"][at, h * G:h * G + G].double()]).max(0).values
            best[-1] = math.inf
            best[:-(-min(case["sinks"], m) // P)] = math.inf
            chosen = torch.sort(best, descending=True, stable=True).indices[:case["picks"]].sort().values
            picks[b, h, :len(chosen)] = chosen.to(torch.int32)
            slots = (chosen[:, None] * P + torch.arange(P, device="cuda")).flatten()
            slots = slots[slots < m]
            for g in group:
                out[at:at + 1, g], lse[at:at + 1, g] = _exact_softmax(s["q"][at:at + 1, g].double(), keys[slots], values[slots])
        at += t
    if case["op"] != "sparse":
        return {"out": out, "lse": lse}
    return {"out": out, "lse": lse, "picks": picks, "k_pages": None, "v_pages": None, "bounds": None}
