"""The paged 8-bit cache, operator by operator: what is timed, in the framework's calls and in plain torch operations.

A sequence's keys and values lie in pages of 128 tokens, 8 bits (e4m3) a value, with one power of two as the scale of each page, KV head
and side; the tokens behind its last full page lie in a bf16 tail.  Every case is one pass through one operator:

  op "grow"      block tables, lengths and the slot of every new row from the sequences' lengths and their numbers of new tokens
  op "store"     new rows into pages and tails, and the same rows read back by their slots as the values that are held
  op "decode"    one query token of each sequence against its pages and tail
  op "prefill"   the new tokens' queries, causal, against everything cached up to them (their own rows included)

A case holds the layer (hq, hkv, d), the sequences (batch; ctx_lo..ctx_hi tokens cached, new_lo..new_hi new ones, spread over the
logarithm by the sequence's number) and the score options: cap (scores capped by cap * tanh(s / cap), 0: not), alibi (a bias of slope
times distance, falling from head to head by the usual powers of two), prefix (that many tokens in front of each sequence see
one another whatever their order).  Layers: the repository's 7B-shaped multi-head and 8B-shaped grouped-query layers and one with heads of 64.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
PAGE = 128

MHA = dict(hq=32, hkv=32, d=128)
GQA = dict(hq=32, hkv=8, d=128)
NARROW = dict(hq=32, hkv=4, d=64)


def _case(op, layer, batch, ctx, new, cap=0.0, alibi=False, prefix=0):
    return dict(op=op, **layer, batch=batch, ctx_lo=ctx[0], ctx_hi=ctx[1], new_lo=new[0], new_hi=new[1], cap=cap, alibi=alibi, prefix=prefix)


def listed():
    return [
        # the tables of one decode step of a serving batch, once for all layers
        dict(name="grow_step_b32", **_case("grow", GQA, 32, (256, 36864), (1, 1))),
        # many prompts of every length admitted at once
        dict(name="grow_prompts_b512", **_case("grow", GQA, 512, (0, 0), (1, 8191))),
        # one token of each of 32 running sequences
        dict(name="store_step_b32", **_case("store", GQA, 32, (256, 36864), (1, 1))),
        # the prompts of a multi-head layer
        dict(name="store_prompts_mha", **_case("store", MHA, 8, (0, 0), (511, 8192))),
        # one short chat: latency
        dict(name="decode_b1_l300", **_case("decode", GQA, 1, (300, 300), (0, 0))),
        # an even batch of a multi-head layer
        dict(name="decode_mha_b8_l4096", **_case("decode", MHA, 8, (4096, 4096), (0, 0))),
        # a serving batch of mixed lengths, capped scores
        dict(name="decode_gqa_b32_ragged_cap", **_case("decode", GQA, 32, (256, 36864), (0, 0), cap=30.0)),
        # one long document
        dict(name="decode_gqa_b1_l131072", **_case("decode", GQA, 1, (131072, 131072), (0, 0))),
        # eight narrow query heads to a KV head, biased by distance
        dict(name="decode_d64_b6_alibi", **_case("decode", NARROW, 6, (77, 20001), (0, 0), alibi=True)),
        # a few drafted or re-submitted tokens behind long contexts
        dict(name="prefill_few_b4", **_case("prefill", GQA, 4, (1000, 30000), (3, 33), alibi=True)),
        # a chunk of a long prompt of a multi-head layer
        dict(name="prefill_mha_8192", **_case("prefill", MHA, 1, (0, 0), (8192, 8192))),
        # prompts of mixed lengths whose first tokens see one another, capped scores
        dict(name="prefill_gqa_b6_prefix_cap", **_case("prefill", GQA, 6, (0, 0), (257, 4001), cap=50.0, prefix=200)),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    layer = rng.choice([MHA, GQA, NARROW, dict(hq=40, hkv=8, d=128), dict(hq=12, hkv=12, d=64)])
    op = rng.choice(["grow", "store", "decode", "decode", "prefill", "prefill"])
    cap, alibi = rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.3
    width = layer["hkv"] * layer["d"]
    if op == "grow":
        batch = _log(rng, 1, 600)
        if rng.random() < 0.5:
            lo = _log(rng, 1, 4000)
            return _case(op, layer, batch, (lo, _log(rng, lo, 36864)), (1, 1))
        hi = _log(rng, 1, 400000 // batch)
        return _case(op, layer, batch, (0, 0), (_log(rng, 1, hi), hi))
    if op == "store":
        if rng.random() < 0.5:
            lo = _log(rng, 1, 4000)
            return _case(op, layer, _log(rng, 1, 64), (lo, _log(rng, lo, 8000)), (1, 1))
        batch = _log(rng, 1, 8)
        hi = _log(rng, 1, min(8192, 20000 * 4096 // (batch * width)))
        return _case(op, layer, batch, (0, 0), (_log(rng, 1, hi), hi))
    if op == "decode":
        batch = _log(rng, 1, 48)
        hi = _log(rng, 1, 131072 * 1024 // (width * batch))
        return _case(op, layer, batch, (_log(rng, 1, hi), hi), (0, 0), cap=cap, alibi=alibi)
    batch, hi = _log(rng, 1, 6), _log(rng, 1, 2000)
    pairs = 400_000_000_000 // (4 * layer["hq"] * layer["d"])             # of a query and a key, for all sequences
    ctx = rng.choice([0, 1]) * _log(rng, 1, max(1, min(8000, (pairs // (batch * hi) - hi) // 2)))
    return _case(op, layer, batch, (ctx, ctx * 2), (_log(rng, 1, hi), hi), cap=cap, alibi=alibi, prefix=rng.choice([0, 0, 33, 500]))


# ---- the case in numbers
def _spread(lo, hi, batch):
    if lo == hi:
        return [lo] * batch
    return [int(round(lo * (hi / lo) ** math.modf((b + 0.5) * 0.6180339887498949)[0])) for b in range(batch)]


def _context(case):
    return _spread(case["ctx_lo"], case["ctx_hi"], case["batch"])


def _new(case):
    return _spread(case["new_lo"], case["new_hi"], case["batch"])


def _slopes(case):
    return [2.0 ** (-8.0 * (h + 1) / case["hq"]) for h in range(case["hq"])]


def _visible(case, before, new):
    """Pairs of one sequence's new tokens and the cached ones that they see."""
    total, pairs = before + new, 0
    prefix = min(case["prefix"], total)
    inside = max(0, min(prefix, total) - before)                        # new tokens that lie in the prefix
    inside = min(inside, new)
    pairs += inside * prefix
    first = before + inside
    n = new - inside
    return pairs + n * first + n * (n + 1) // 2


def work(case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    width, rows, total = hkv * d, sum(_new(case)), sum(_context(case)) + sum(_new(case))
    full = sum((c + n) // PAGE * PAGE for c, n in zip(_context(case), _new(case)))
    cached = 2 * width * full + 4 * width * (total - full) + 2 * hkv * (full // PAGE)
    if case["op"] == "grow":
        pages = sum((c + n) // PAGE - c // PAGE for c, n in zip(_context(case), _new(case)))
        return {"bytes": 8 * rows + 8 * pages + 16 * case["batch"], "flops": 0}
    if case["op"] == "store":
        done = sum(min(n, (c + n) // PAGE * PAGE - c) for c, n in zip(_context(case), _new(case)) if (c + n) // PAGE > c // PAGE)
        held = 2 * width * done + 4 * width * (rows - done)
        return {"bytes": 4 * width * rows + 2 * held + 4 * width * rows + 4 * rows, "flops": 0}
    if case["op"] == "decode":
        return {"bytes": cached + 4 * case["batch"] * hq * d, "flops": 4 * hq * d * total}
    pairs = sum(_visible(case, c, n) for c, n in zip(_context(case), _new(case)))
    return {"bytes": cached + 4 * rows * hq * d, "flops": 4 * hq * d * pairs}


# ---- inputs
def _inputs(case, seed):
    """Everything random, the same on every side: rows of all tokens (cached ones first, sequence by sequence), queries, the pool's order."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    ctx, new = _context(case), _new(case)
    hkv, d = case["hkv"], case["d"]
    pages = sum((c + n) // PAGE for c, n in zip(ctx, new)) + 8
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    x = dict(order=order)
    if case["op"] == "grow":
        return x

    def rows(count, channels):
        out = torch.empty(count, hkv, d, dtype=torch.bfloat16, device=DEV)
        for i in range(0, count, 65536):
            part = out[i:i + 65536]
            part.copy_(torch.randn(part.shape, generator=gen, device=DEV) * channels)
        return out

    channels = torch.exp(0.5 * torch.randn(hkv, d, generator=gen, device=DEV))      # keys have channels of their own size
    total = sum(ctx) + sum(new)
    x["k"], x["v"] = rows(total, channels), rows(total, 1.0)
    queries = case["batch"] if case["op"] == "decode" else sum(new)
    x["q"] = torch.randn(queries, case["hq"], d, generator=gen, device=DEV).to(torch.bfloat16)
    return x


def _split(case, rows):
    """All tokens' rows to (cached ones, new ones), each packed by sequence."""
    old, new, at = [], [], 0
    for c, n in zip(_context(case), _new(case)):
        old.append(rows[at:at + c])
        new.append(rows[at + c:at + c + n])
        at += c + n
    return torch.cat(old), torch.cat(new)


def _table(case, order):
    """Block table of the cached tokens and the stack of free pages, its top at the end, with its height."""
    full = [c // PAGE for c in _context(case)]
    width = max((c + n) // PAGE for c, n in zip(_context(case), _new(case))) + 1
    table = torch.full((case["batch"], width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, f in enumerate(full):
        table[b, :f] = order[at:at + f]
        at += f
    free = order.new_zeros(order.numel())
    free[:order.numel() - at] = order[at:].flip(0)
    return table, free, order.numel() - at


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    x = _inputs(case, seed)
    table, free, n_free = _table(case, x["order"])
    st = dict(case=case, table=table, free=free, n_free=_int([n_free]), len0=_int(_context(case)), n_new=_int(_new(case)),
              rows=sum(_new(case)))
    if case["op"] != "grow":
        st["q"] = x["q"]
        st["slopes"] = torch.tensor(_slopes(case), dtype=torch.float32, device=DEV) if case["alibi"] else None
        old, new = zip(*(_split(case, x[s]) for s in "kv"))
        st["new"] = new
        st["prefix"] = _int([case["prefix"]] * case["batch"]) if case["prefix"] else None
        (_prepare_own if own else _prepare_plain)(case, st, old)
    elif own:
        _prepare_own(case, st, None)
    torch.cuda.synchronize()
    return st


# ---- the framework's calls
def _prepare_own(case, st, old):
    from paper_2603_22910_amd import binding as ek
    batch, rows = case["batch"], st["rows"]
    st["shape"] = ek.make_shape(case["hq"], case["hkv"], case["d"], 0, "bf16")
    plan = lambda n: ek.PagePlan(torch.empty(ek.page_plan_bytes(batch), dtype=torch.uint8, device=DEV), batch, n)
    st["plan"] = plan(max(1, rows))
    st["len1"], st["n_free1"] = torch.empty_like(st["len0"]), torch.empty_like(st["n_free"])
    st["slot"], st["pos"] = (torch.empty(max(1, rows), dtype=torch.int32, device=DEV) for _ in range(2))
    if case["op"] == "grow":
        st["pages"] = ek.PageTable(st["table"], st["len0"], st["free"], st["n_free"])
        return
    cache = st["cache"] = ek.PageCache.empty(st["shape"], batch, st["free"].numel(), DEV)
    pages = st["pages"] = ek.PageTable(st["table"], torch.zeros_like(st["len0"]), st["free"], st["n_free"])
    cached = sum(_context(case))
    if cached:                                   # the cached tokens come the way they come in a program: as new ones
        before = plan(cached)
        pages.free_list, pages.n_free = _all_free(st), _int([st["free"].numel()])
        ek.pages_grow(st["shape"], pages, st["len0"], before)
        ek.page_append(st["shape"], pages, cache, before, old[0], old[1])
        st["plan"] = before
    if rows:
        st["plan"] = plan(rows)
        ek.pages_grow(st["shape"], pages, st["n_new"], st["plan"], row_slot=st["slot"], row_pos=st["pos"])
        if case["op"] == "prefill":
            ek.page_append(st["shape"], pages, cache, st["plan"], st["new"][0], st["new"][1])
    width = case["hkv"] * case["d"]
    if case["op"] == "store":
        st["out"] = [torch.empty(rows, width, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    else:
        st["out"] = [torch.empty_like(st["q"]), torch.empty(st["q"].shape[:2], dtype=torch.float32, device=DEV)]
        nbytes = ek.page_workspace_bytes(st["shape"], batch, st["plan"].max_rows if case["op"] == "prefill" else 0)
        st["ws"] = torch.empty(nbytes, dtype=torch.uint8, device=DEV)


def _all_free(st):
    """The whole pool as a stack from which the cached tokens' pages come off in the order of the table."""
    used = st["table"][st["table"] >= 0]
    rest = st["free"][:int(st["n_free"])]
    return torch.cat([rest, used.flip(0)])


def _run_own(st):
    from paper_2603_22910_amd import binding as ek
    op, case = st["case"]["op"], st["case"]
    if op == "grow":
        ek.pages_grow(st["shape"], st["pages"], st["n_new"], st["plan"], seq_len_out=st["len1"], n_free_out=st["n_free1"],
                      row_slot=st["slot"], row_pos=st["pos"])
        return [st["len1"], st["n_free1"], st["table"], st["plan"].row_start, st["slot"], st["pos"]]
    if op == "store":
        ek.page_append(st["shape"], st["pages"], st["cache"], st["plan"], st["new"][0], st["new"][1])
        ek.page_read(st["shape"], st["pages"], st["cache"], st["slot"], st["out"][0], st["out"][1])
        return st["out"]
    if op == "decode":
        ek.page_decode_attn(st["shape"], st["pages"], st["cache"], st["plan"], st["q"], st["out"][0], st["out"][1], st["ws"],
                            softcap=case["cap"], slopes=st["slopes"])
    else:
        ek.page_prefill_attn(st["shape"], st["pages"], st["cache"], st["plan"], st["q"], st["out"][0], st["out"][1], st["ws"],
                             softcap=case["cap"], slopes=st["slopes"], prefix_len=st["prefix"])
    return st["out"]


# ---- the plain form
def _quantise(blocks):
    """[n, 128, hkv, d] rows -> e4m3 codes of the same shape and the scales [n, 1, hkv, 1], powers of two."""
    x = _finite(blocks.float())
    amax = x.abs().amax(dim=(1, 3), keepdim=True)
    mantissa, exponent = torch.frexp(amax)
    e = torch.clamp(exponent - torch.where(mantissa > 0.875, 8, 9), min=-100)
    scale = torch.ldexp(torch.ones_like(amax), e)
    return (x * torch.ldexp(torch.ones_like(amax), -e)).to(torch.float8_e4m3fn), scale


def _finite(x):
    top = 1.75 * 2.0 ** 127                                       # the largest number of a page
    return torch.where(torch.isnan(x), 0.0, x).clamp(-top, top)


def _prepare_plain(case, st, old):
    """Pages and tails of the cached tokens in the order of their rows, and which rows the new tokens' blocks take."""
    hkv, d, batch = case["hkv"], case["d"], case["batch"]
    pages = st["free"].numel()
    st["codes"] = [torch.zeros(pages, PAGE, hkv, d, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2)]
    st["scale"] = [torch.ones(pages, 1, hkv, 1, device=DEV) for _ in range(2)]
    st["tail"] = [torch.zeros(batch * PAGE, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    free = st["free"].tolist()
    top, table = int(st["n_free"]), st["table"].tolist()
    for which, rows in ((0, None), (1, None)):
        at = 0
        for b, c in enumerate(_context(case)):
            f = c // PAGE
            for i in range(0, f, 64):
                n = min(64, f - i)
                codes, scale = _quantise(old[which][at + i * PAGE:at + (i + n) * PAGE].view(n, PAGE, hkv, d))
                index = st["table"][b, i:i + n].long()
                st["codes"][which].view(torch.uint8)[index] = codes.view(torch.uint8)
                st["scale"][which][index] = scale
            st["tail"][which][b * PAGE:b * PAGE + c - f * PAGE] = _finite(old[which][at + f * PAGE:at + c].float()).bfloat16()
            at += c
    block_rows, block_page, tail_from, tail_to, slots, at = [], [], [], [], [], 0
    for b, (c, n) in enumerate(zip(_context(case), _new(case))):
        source = lambda p: b * PAGE + p % PAGE if p < c else batch * PAGE + at + p - c
        for blk in range(c // PAGE, (c + n) // PAGE):
            top -= 1
            table[b][blk] = free[top]
            block_page.append(free[top])
            block_rows.append([source(p) for p in range(blk * PAGE, (blk + 1) * PAGE)])
        for p in range(max(c, (c + n) // PAGE * PAGE), c + n):
            tail_from.append(at + p - c)
            tail_to.append(b * PAGE + p % PAGE)
        for p in range(c, c + n):
            slots.append(table[b][p // PAGE] * PAGE + p % PAGE if p < (c + n) // PAGE * PAGE else -1 - (b * PAGE + p % PAGE))
        at += n
    index = lambda v: torch.tensor(v, dtype=torch.int64, device=DEV)
    st["table"] = _int(table)
    st["block_rows"], st["block_page"] = index(block_rows).view(-1, PAGE), index(block_page)
    st["tail_from"], st["tail_to"], st["slots"] = index(tail_from), index(tail_to), index(slots)
    if case["op"] == "prefill":
        _store_plain(st)


def _store_plain(st):
    """The new rows into pages and tails."""
    for which in range(2):
        rows = st["new"][which]
        if st["block_page"].numel():
            every = torch.cat([st["tail"][which], rows])
            for i in range(0, st["block_page"].numel(), 256):
                codes, scale = _quantise(every[st["block_rows"][i:i + 256]])
                st["codes"][which].view(torch.uint8)[st["block_page"][i:i + 256]] = codes.view(torch.uint8)
                st["scale"][which][st["block_page"][i:i + 256]] = scale
        st["tail"][which][st["tail_to"]] = _finite(rows[st["tail_from"]].float()).bfloat16()


def _read_plain(st):
    case, slots, out = st["case"], st["slots"], []
    page, tail = torch.clamp(slots, min=0), torch.clamp(-1 - slots, min=0)
    for which in range(2):
        got = torch.empty(slots.numel(), case["hkv"], case["d"], dtype=torch.bfloat16, device=DEV)
        for i in range(0, slots.numel(), 16384):
            at = page[i:i + 16384]
            codes = st["codes"][which].view(torch.uint8)[at // PAGE, at % PAGE].view(torch.float8_e4m3fn)
            held = codes.float() * st["scale"][which][at // PAGE, 0]
            got[i:i + 16384] = torch.where((slots[i:i + 16384] >= 0)[:, None, None], held.bfloat16(), st["tail"][which][tail[i:i + 16384]])
        out.append(got.view(slots.numel(), -1))
    return out


def _sequence(st, which, b, length):
    """Keys or values [hkv, length, d] of one sequence in 32 bits."""
    full = length // PAGE
    index = st["table"][b, :full].long()
    codes = st["codes"][which].view(torch.uint8)[index].view(torch.float8_e4m3fn)
    held = (codes.float() * st["scale"][which][index]).flatten(0, 1)
    tail = st["tail"][which][b * PAGE:b * PAGE + length % PAGE].float()
    return torch.cat([held, tail]).transpose(0, 1).contiguous()


def _attend(case, slopes, q, k, v, positions):
    """q [n, hq, d] at the given positions; k, v [hkv, length, d]: outputs [n, hq, d] and the logarithms of the sums [n, hq]."""
    n, hq, d = q.shape
    hkv, length, _ = k.shape
    g = hq // hkv
    keys = torch.arange(length, device=DEV)
    seen = (keys[None] <= positions[:, None]) | (keys < case["prefix"])[None]
    away = (keys[None] - positions[:, None]).float()
    out, lse = torch.empty(n, hq, d, device=DEV), torch.empty(n, hq, device=DEV)
    kv_heads = max(1, (1 << 28) // max(1, n * g * length))              # so many at once
    for a in range(0, hkv, kv_heads):
        b = min(hkv, a + kv_heads)
        heads = slice(a * g, b * g)
        s = torch.matmul(q[:, heads].float().view(n, b - a, g, d).permute(1, 2, 0, 3).reshape(b - a, g * n, d),
                         k[a:b].transpose(1, 2).contiguous()) * (1.0 / math.sqrt(d))
        if case["cap"]:
            s = case["cap"] * torch.tanh(s / case["cap"])
        s = s.view(b - a, g, n, length)
        if slopes is not None:
            s = s + slopes[heads].view(b - a, g, 1, 1) * away
        s = torch.where(seen, s, -torch.inf)
        top = s.amax(dim=3, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(dim=3, keepdim=True)
        o = torch.matmul(p.view(b - a, g * n, length), v[a:b]).view(b - a, g, n, d) / total
        out[:, heads] = o.permute(2, 0, 1, 3).reshape(n, (b - a) * g, d)
        lse[:, heads] = (top + torch.log(total)).squeeze(3).permute(2, 0, 1).reshape(n, (b - a) * g)
    return out.to(torch.bfloat16), lse


def _run_plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "grow":
        return _grow_plain(st)
    if op == "store":
        _store_plain(st)
        return _read_plain(st)
    out, lse, at = [], [], 0
    for b, (c, n) in enumerate(zip(_context(case), _new(case))):
        length = c + n
        k, v = _sequence(st, 0, b, length), _sequence(st, 1, b, length)
        first, count = (length - 1, 1) if op == "decode" else (c, n)
        for i in range(0, count, 2048):
            m = min(2048, count - i)
            o, l = _attend(case, st["slopes"], st["q"][at + i:at + i + m], k, v, torch.arange(first + i, first + i + m, device=DEV))
            out.append(o)
            lse.append(l)
        at += count
    return [torch.cat(out), torch.cat(lse)]


def _grow_plain(st):
    len0, n_new, table = st["len0"], st["n_new"], st["table"]
    len1 = len0 + n_new
    old, new = len0 // PAGE, len1 // PAGE
    count = new - old
    base = torch.cumsum(count, 0) - count
    nth = torch.arange(table.shape[1], device=DEV, dtype=torch.int32)[None] - old[:, None]
    fresh = (nth >= 0) & (nth < count[:, None])
    at = torch.clamp(st["n_free"] - 1 - (base[:, None] + nth), min=0)
    table = torch.where(fresh, st["free"][at.long()], table)
    row_start = torch.zeros(len0.numel() + 1, dtype=torch.int32, device=DEV)
    row_start[1:] = torch.cumsum(n_new, 0)
    rows = torch.arange(st["rows"], device=DEV, dtype=torch.int32)
    b = torch.searchsorted(row_start, rows, right=True) - 1
    pos = len0[b] + rows - row_start[b]
    page = table[b, torch.clamp(pos // PAGE, max=table.shape[1] - 1).long()]
    slot = torch.where(pos // PAGE < new[b], page * PAGE + pos % PAGE, -1 - (b * PAGE + pos % PAGE))
    return [len1, (st["n_free"] - count.sum()).int(), table, row_start, slot.int(), pos.int()]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definition in 64 bits
def _held(rows):
    """What a sequence's rows [length, hkv, d] are held as, in 64 bits."""
    x = rows.double()
    x = torch.nan_to_num(x, nan=0.0).clamp(-448.0 * 2.0 ** 119, 448.0 * 2.0 ** 119)
    full = x.shape[0] // PAGE * PAGE
    blocks = x[:full].view(-1, PAGE, x.shape[1], x.shape[2])
    largest = blocks.abs().amax(dim=(1, 3), keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp(largest, min=1e-300) / 448.0))
    e = torch.where(largest > 448.0 * torch.exp2(e), e + 1, e)
    e = torch.where(largest <= 448.0 * torch.exp2(e - 1), e - 1, e)
    scale = torch.exp2(torch.clamp(e, min=-100.0))
    y = blocks / scale
    step = torch.exp2(torch.clamp(torch.frexp(y)[1] - 1, min=-6).double() - 3)      # of e4m3: three bits behind the leading one
    held = torch.where(y == 0, 0.0, torch.round(y / step) * step) * scale
    return torch.cat([held.view(full, x.shape[1], x.shape[2]), x[full:]])


def exact(case, seed):
    x = _inputs(case, seed)
    ctx, new = _context(case), _new(case)
    if case["op"] == "grow":
        return _exact_grow(case, x["order"])
    hkv, d, g = case["hkv"], case["d"], case["hq"] // case["hkv"]
    outs, sums, kept, at, row = [], [], ([], []), 0, 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        k, v = (_held(x[s][at:at + c + n]) for s in "kv")
        at += c + n
        if case["op"] == "store":
            kept[0].append(k[c:].reshape(n, hkv * d))
            kept[1].append(v[c:].reshape(n, hkv * d))
            continue
        count, first = (1, c + n - 1) if case["op"] == "decode" else (n, c)
        q = x["q"][row:row + count].double()
        row += count
        keys = torch.arange(c + n, device=DEV, dtype=torch.float64)
        out, total = torch.empty(count, case["hq"], d, dtype=torch.float64, device=DEV), torch.empty(count, case["hq"], dtype=torch.float64, device=DEV)
        step = max(1, (1 << 25) // (c + n))
        for i in range(0, count, step):
            pos = first + torch.arange(i, min(count, i + step), device=DEV, dtype=torch.float64)[:, None]
            hidden = (keys > pos) & (keys >= case["prefix"])
            for h in range(case["hq"]):
                s = q[i:i + step, h] @ k[:, h // g].T / math.sqrt(d)
                if case["cap"]:
                    s = torch.tanh(s / case["cap"]) * case["cap"]
                if case["alibi"]:
                    s = s - (pos - keys) * _slopes(case)[h]
                s = s.masked_fill(hidden, -math.inf)
                z = torch.logsumexp(s, dim=1, keepdim=True)
                total[i:i + step, h] = z[:, 0]
                out[i:i + step, h] = torch.exp(s - z) @ v[:, h // g]
        outs.append(out)
        sums.append(total)
    if case["op"] == "store":
        return [torch.cat(kept[0]), torch.cat(kept[1])]
    return [torch.cat(outs), torch.cat(sums)]


def _exact_grow(case, order):
    table, free, n_free = (t.cpu().numpy() if isinstance(t, torch.Tensor) else t for t in _table(case, order))
    table, slots, positions, starts = table.copy(), [], [], [0]
    lengths = []
    for b, (c, n) in enumerate(zip(_context(case), _new(case))):
        for blk in range(c // PAGE, (c + n) // PAGE):
            n_free -= 1
            table[b, blk] = free[n_free]
        pos = np.arange(c, c + n)
        done = pos < (c + n) // PAGE * PAGE
        slots.append(np.where(done, table[b, np.where(done, pos // PAGE, 0)].astype(np.int64) * PAGE + pos % PAGE, -1 - (b * PAGE + pos % PAGE)))
        positions.append(pos)
        starts.append(starts[-1] + n)
        lengths.append(c + n)
    return [_int(lengths), _int([n_free]), _int(table.tolist()), _int(starts), _int(np.concatenate(slots).tolist()), _int(np.concatenate(positions).tolist())]
