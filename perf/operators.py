"""Softmax attention over a paged key/value cache, as cases that can be timed: what a serving program asks of it next to the
hybrid attention of this library.  Layers that keep every token, or a sliding window and a few first tokens, hold their
keys and values in pages of a shared pool instead of a ring; a cache that may not grow gives up the slots whose accumulated
attention weight is least.

  op        "decode":  one new token per sequence is stored and attends to the sequence's cache; tracked: the weights that it
                       gives the slots are added to the cache's account of them
            "prefill": a prompt's (or a further turn's) tokens are stored and attend, each to the tokens up to itself
            "prompt":  prefill, and the weights that all of the call's tokens give the slots are added to the account
            "evict":   every (sequence, KV head) keeps `budget` slots: the first tokens, the newest tokens, and those of the
                       largest weight; the rows kept beyond the budget move into the slots given up
  heads, kv_heads, dim, dtype, page (tokens of a page), batch
  context   tokens in the cache before the pass (of the longest sequence)
  tokens    new tokens of the pass (of the longest sequence)
  ragged    the sequences' lengths differ
  window    newest tokens that a token sees, itself among them (-1: all);  sinks: first tokens that stay visible
  tracked   decode: with the account of weights
  budget, recent   evict: slots kept per sequence; newest tokens that are kept whatever their weight

With `own` false, `run` computes all this from elementary torch operations in fp32."""
import math

import torch

own = False

_LLAMA = dict(heads=32, kv_heads=8, dim=128, dtype="bf16", page=64)
_TINY = dict(heads=4, kv_heads=4, dim=64, dtype="f32", page=16)
_PLAIN = dict(batch=1, context=0, tokens=0, ragged=False, window=-1, sinks=0, tracked=False, budget=0, recent=0)


def _case(name, op, shape, **kw):
    return dict(_PLAIN, name=name, op=op, **shape) | kw


def listed():
    return [
        # The smallest call: one fp32 layer of 4 heads behind a 512-token prompt.
        _case("decode_tiny_f32", "decode", _TINY, context=512, tokens=1),
        # Interactive decode of one 32K-token sequence that keeps every token.
        _case("decode_b1_32k", "decode", _LLAMA, context=32768, tokens=1),
        # A serving batch of different lengths, a window of 1024 tokens and four first ones.
        _case("decode_sinks_b16_16k", "decode", _LLAMA, batch=16, context=16384, tokens=1, ragged=True, window=1024, sinks=4),
        # Long documents: four sequences of 128K tokens.
        _case("decode_b4_128k", "decode", _LLAMA, batch=4, context=131072, tokens=1),
        # The step of a cache that gives up slots by weight: the step's weights are added to the account.
        _case("decode_tracked_b8_8k", "decode", _LLAMA, batch=8, context=8192, tokens=1, ragged=True, tracked=True),
        # One long prompt, a length that is no multiple of any tile.
        _case("prefill_b1_8k", "prefill", _LLAMA, tokens=8001),
        # A batch of prompts of different lengths, a window and first tokens.
        _case("prefill_sinks_b8_2k", "prefill", _LLAMA, batch=8, tokens=2048, ragged=True, window=256, sinks=4),
        # A further turn of long conversations: 1000 tokens each on top of 128K.
        _case("prefill_turn_b4_128k", "prefill", _LLAMA, batch=4, context=131072, tokens=1000),
        # A small fp32 prompt whose weights decide what is kept of it ...
        _case("prompt_tiny_f32", "prompt", _TINY, tokens=512, window=64, sinks=1),
        # ... and two long ones.
        _case("prompt_b2_4k", "prompt", _LLAMA, batch=2, tokens=4096, ragged=True),
        # After a long prompt an eighth of it is kept ...
        _case("evict_b1_32k", "evict", _LLAMA, context=32768, budget=4096, recent=256, sinks=4),
        # ... and from then on every step gives up one slot of each sequence.
        _case("evict_step_b16_4k", "evict", _LLAMA, batch=16, context=4097, budget=4096, recent=256, sinks=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: every operator, fp32 and bf16, 1 to 8 KV heads with 1 to 8 query heads each, 1 to 16 sequences of
    one token to 64K, pages of 16 to 128 tokens, windows from one token to all of them."""
    op = rng.choice(["decode", "decode", "prefill", "prefill", "prompt", "evict"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8])
    shape = dict(heads=kv_heads * group, kv_heads=kv_heads, dim=rng.choice([64, 128]), dtype=dtype, page=rng.choice([16, 32, 64, 128]))
    batch = _log_int(rng, 1, 16)
    c = _case("", op, shape, batch=batch, ragged=rng.random() < 0.7)
    small = dtype == "f32"
    if rng.random() < 0.5:
        c.update(window=_log_int(rng, 1, 4096), sinks=rng.choice([0, 1, 4, 100]))
    if op == "decode":
        c.update(tokens=1, context=_log_int(rng, 1, (16384 if small else 65536) // batch), tracked=rng.random() < 0.4)
    elif op == "evict":
        c.update(context=_log_int(rng, 64, 65536 // batch), window=-1, sinks=rng.choice([0, 1, 4]))
        c["budget"] = max(16, c["context"] - 1 if rng.random() < 0.4 else _log_int(rng, 16, c["context"]))
        c["recent"] = rng.randint(0, c["budget"] // 2)
    else:
        c.update(tokens=max(1, _log_int(rng, 2, 1000 if small else 8000) // batch))
        if rng.random() < 0.5:
            c["context"] = _log_int(rng, 1, (4096 if small else 32768) // batch)
    del c["name"]
    return c


def _lengths(case):
    """Per sequence: tokens in the cache before the pass, new tokens."""
    before, new = [], []
    for b in range(case["batch"]):
        part = 2000 if case["ragged"] else 0
        before.append(case["context"] - (b * 617 % 1000) * case["context"] // part if part else case["context"])
        new.append(max(1, case["tokens"] - (b * 389 % 1000) * case["tokens"] // part) if part and case["tokens"] else case["tokens"])
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
    starts = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
    rows = sum(new)
    s = dict(case=case, table=table, starts=starts, before=torch.tensor(before, device="cuda", dtype=torch.int32),
             lens=torch.tensor(lens, device="cuda", dtype=torch.int32), most=max(lens), most_new=max(new),
             k_pages=normal(1, pages, Hkv, page, d), v_pages=normal(1, pages, Hkv, page, d))
    if case["op"] != "evict":
        s.update(q=normal(rows, H, d, scale=2.0), k=normal(rows, Hkv, d), v=normal(rows, Hkv, d))
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(rows, H, device="cuda")
    if case["tracked"] or case["op"] in ("prompt", "evict"):
        # Weights that a cache has gathered: a few large, many small, some tokens never seen.
        shape = (B, Hkv, cols * page)
        w = torch.randn(shape, generator=gen, device="cuda").mul_(1.5).exp_()
        s["weight"] = torch.where(torch.rand(shape, generator=gen, device="cuda") < 0.01, 0.0, w)
        # After earlier slots were given up, half of the sequence's tokens are left, in any order behind the first few.
        seen = s["lens"] if case["op"] == "prompt" else s["lens"] * 2
        order = torch.rand(shape, generator=gen, device="cuda")
        order = torch.where(torch.arange(shape[2], device="cuda") < s["lens"][:, None, None], order, 2.0)
        place = order.argsort(dim=2).argsort(dim=2)
        s["pos"] = torch.where(place < case["sinks"], place, place + (seen - s["lens"])[:, None, None]).to(torch.int32)
        s["seen"] = seen
        s["weight_out"], s["pos_out"] = torch.zeros_like(s["weight"]), torch.zeros_like(s["pos"])
        s["new_lens"] = torch.zeros_like(s["lens"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2607_24788_b200 import glide
        s["cache"] = glide.GlidePaged(s["k_pages"], s["v_pages"], case["heads"], case["batch"], s["table"].shape[1] * case["page"])
    return s


# ---- the calls of the framework -------------------------------------------------------------------


def _run_own(s):
    case, cache = s["case"], s["cache"]
    mask = dict(window=case["window"], n_sink=case["sinks"])
    if case["op"] == "evict":
        cache.glide_paged_evict(s["table"], s["lens"], s["seen"], s["weight"], s["pos"], case["budget"], s["new_lens"], recent=case["recent"],
                                n_sink=case["sinks"], weight_out=s["weight_out"], pos_out=s["pos_out"])
        return {n: s[n] for n in ("k_pages", "v_pages", "weight_out", "pos_out", "new_lens")}
    if case["op"] == "decode":
        if case["tracked"]:
            cache.glide_paged_decode(s["table"], s["lens"], s["q"], s["k"], s["v"], s["out"], weight=s["weight"], pos=s["pos"], seen=s["seen"], **mask)
            return {n: s[n] for n in ("out", "k_pages", "v_pages", "weight", "pos")}
        cache.glide_paged_decode(s["table"], s["lens"], s["q"], s["k"], s["v"], s["out"], **mask)
        return {n: s[n] for n in ("out", "k_pages", "v_pages")}
    if case["op"] == "prefill":
        cache.glide_paged_prefill(s["table"], s["lens"], s["starts"], s["q"], s["k"], s["v"], s["out"], **mask)
        return {n: s[n] for n in ("out", "k_pages", "v_pages")}
    cache.glide_paged_prefill(s["table"], s["lens"], s["starts"], s["q"], s["k"], s["v"], s["out"], lse=s["lse"], weight=s["weight"], pos=s["pos"],
                              seen=s["seen"], **mask)
    cache.glide_paged_weights(s["table"], s["lens"], s["starts"], s["q"], s["lse"], s["weight"], **mask)
    return {n: s[n] for n in ("out", "lse", "k_pages", "v_pages", "weight", "pos")}


# ---- the plain forms ------------------------------------------------------------------------------


def _place(s, seq, slot):
    """Page and offset of slots of sequences."""
    page = s["case"]["page"]
    return s["table"][seq, slot // page].long(), slot % page


def _store(s):
    """The new tokens' keys and values into their slots; the account of a new slot starts at 0."""
    row = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(s["starts"][1:].contiguous(), row.to(torch.int32), right=True)
    at = row - s["starts"][seq]
    slot = s["before"][seq] + at
    page, off = _place(s, seq, slot)
    s["k_pages"][0][page, :, off] = s["k"]
    s["v_pages"][0][page, :, off] = s["v"]
    if "weight" in s:
        s["weight"][seq, :, slot] = 0.0
        s["pos"][seq, :, slot] = (s["seen"] - s["lens"])[seq, None] + slot[:, None].to(torch.int32)
    return seq, at


def _attend(s, seq, at):
    """Outputs and logarithms of the row sums of every new token, its weights summed per slot where the cache keeps account."""
    case = s["case"]
    B, H, Hkv, d, T, w, n0 = case["batch"], case["heads"], case["kv_heads"], case["dim"], s["most_new"], case["window"], case["sinks"]
    G, most = H // Hkv, s["most"]
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
    step = max(1, min(Hkv, (2 << 30) // (B * G * T * slot.shape[1])))
    for h in range(0, Hkv, step):
        heads = slice(h, h + step)
        k, v = (x[0].permute(0, 2, 1, 3)[page, off, heads].float().transpose(1, 2) for x in (s["k_pages"], s["v_pages"]))
        n = k.shape[1]
        x = torch.matmul(q[:, heads], k.transpose(-1, -2)).view(B, n, G, T, -1).masked_fill_(~sees, -math.inf)
        top = x.amax(-1, keepdim=True)
        p = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
        total = p.sum(-1, keepdim=True)
        lse = (top + total.log()).squeeze(-1)
        total = torch.where(total == 0.0, 1.0, total)
        o = torch.matmul(p.view(B, n, G * T, -1), v).view(B, n, G, T, d) / total
        s["out"].view(-1, Hkv, G, d)[:, heads] = o.permute(0, 3, 1, 2, 4)[seq, at].to(s["out"].dtype)
        s["lse"].view(-1, Hkv, G)[:, heads] = lse.permute(0, 3, 1, 2)[seq, at]
        if "weight" in s:
            live = (torch.arange(T, device="cuda") < (s["lens"] - s["before"])[:, None])[:, None, None, :, None]
            given = p.div_(total).masked_fill_(~live, 0.0).sum((2, 3)).masked_fill_(~there[:, None], 0.0)
            s["weight"][:, heads].scatter_add_(2, slot.clamp(max=most - 1)[:, None].expand(B, n, -1), given)


def _evict(s):
    case = s["case"]
    B, Hkv, most, budget = case["batch"], case["kv_heads"], s["most"], case["budget"]
    lens, slot = s["lens"][:, None, None], torch.arange(most, device="cuda")
    pos = s["pos"][..., :most]
    safe = (pos < case["sinks"]) | (pos >= s["seen"][:, None, None] - case["recent"])
    key = torch.where(safe | (slot >= lens), math.inf, s["weight"][..., :most])
    rank = key.argsort(dim=2, stable=True).argsort(dim=2)                            # equal weights: the lowest slot goes first
    gone = rank < (lens - budget)
    kept = lens.clamp(max=budget)
    s["new_lens"].copy_(kept[:, 0, 0])
    b, h, dst = (gone & (slot < kept)).nonzero(as_tuple=True)
    _, _, src = (~gone & (slot >= kept) & (slot < lens)).nonzero(as_tuple=True)
    page_to, off_to = _place(s, b, dst)
    page_of, off_of = _place(s, b, src)
    for x in (s["k_pages"], s["v_pages"]):
        x[0][page_to, h, off_to] = x[0][page_of, h, off_of]
    there = torch.arange(s["weight"].shape[2], device="cuda") < kept
    for name in ("weight", "pos"):
        s[name + "_out"].copy_(torch.where(there, s[name], s[name + "_out"]))
        s[name + "_out"][b, h, dst] = s[name][b, h, src]


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    if op == "evict":
        _evict(s)
        return {n: s[n] for n in ("k_pages", "v_pages", "weight_out", "pos_out", "new_lens")}
    seq, at = _store(s)
    _attend(s, seq, at)
    names = ["out"] + ["lse"] * (op == "prompt") + ["k_pages", "v_pages"] + ["weight", "pos"] * ("weight" in s)
    return {n: s[n] for n in names}


def work(case):
    """One pass: the visible slots' keys and values, the new tokens' tensors and the account read once, the new rows, outputs and
    the account written once; multiply-adds of the two products (a third one where a prompt's weights are summed, which need the
    row sums first).  evict: every slot's weight and position, and the kept ones' written, the rows that have to move read and written."""
    H, Hkv, d = case["heads"], case["kv_heads"], case["dim"]
    elem = 4 if case["dtype"] == "f32" else 2
    before, new = _lengths(case)
    byts = flops = 0
    for n, t in zip(before, new):
        if case["op"] == "evict":
            kept = min(n, case["budget"])
            # of the kept slots those behind the budget move: of slots in any order (n - kept) / n of them
            byts += Hkv * (8 * n + 8 * kept + 4 * kept * (n - kept) // n * d * elem)
            continue
        w = n + t if case["window"] < 0 else case["window"]
        first = min(case["sinks"], n + t)
        old = min(n, w - 1 if w else 0)
        old += max(0, min(first, n - old))
        byts += 2 * (old + 2 * t) * Hkv * d * elem + 2 * t * H * d * elem
        pairs = sum(min(i, w) + min(first, max(0, i - w)) for i in range(n + 1, n + t + 1))
        flops += 4 * H * d * pairs
        if case["op"] == "prompt":
            flops += 2 * H * d * pairs
            byts += (8 * t + 8 * (n + t)) * Hkv + 4 * t * H
        elif case["tracked"]:
            byts += 8 * (old + t) * Hkv + 4 * Hkv
    return dict(bytes=byts, flops=flops)


def exact(case, seed):
    """The attention's definition, sequence by sequence and head by head, in 64 bits.  Rows that are only moved have no such value."""
    if case["op"] == "evict":
        return None
    s = _inputs(case, seed)
    H, Hkv, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    G = H // Hkv
    before, new = _lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    weight = s["weight"].double() if "weight" in s else None
    at = 0
    for b in range(case["batch"]):
        n, t = before[b], new[b]
        pages = s["table"][b, :-(-(n + t) // page)].long()
        i = torch.arange(n, n + t, device="cuda")[:, None]
        j = torch.arange(n + t, device="cuda")[None]
        hidden = j > i
        if case["window"] >= 0:
            hidden = hidden | ((j <= i - case["window"]) & (j >= case["sinks"]))
        if weight is not None:
            weight[b, :, n:n + t] = 0.0
        for h in range(Hkv):
            keys = torch.cat([s["k_pages"][0, pages, h].reshape(-1, d)[:n], s["k"][at:at + t, h]]).double()
            values = torch.cat([s["v_pages"][0, pages, h].reshape(-1, d)[:n], s["v"][at:at + t, h]]).double()
            for g in range(h * G, h * G + G):
                x = s["q"][at:at + t, g].double() @ keys.T / math.sqrt(d)
                x.masked_fill_(hidden, -math.inf)
                total = torch.logsumexp(x, 1)
                p = torch.exp(x - torch.where(total == -math.inf, 0.0, total)[:, None])
                out[at:at + t, g] = p @ values
                lse[at:at + t, g] = total
                if weight is not None:
                    weight[b, h, :n + t] += p.sum(0)
        at += t
    got = {"out": out, "k_pages": None, "v_pages": None}
    if case["op"] == "prompt":
        got["lse"] = lse
    if weight is not None:
        got.update(weight=weight, pos=None)
    return got
