"""The operators around an 8-bit key/value cache, measured: block tables from request lengths, the rotary append, and the
attention that reads the cache.

    listed()  the cases;  draw(rng)  one more case of the same ranges
    prepare(case, seed)  inputs and state on the GPU;  run(state)  one pass of one operator, outputs whole
    work(case)  bytes and operations of a pass;  exact(case, seed)  the outputs from the definitions in 64 bits

`own` is set from outside: false runs the plain forms below, true the calls of the library.

A case describes a batch of requests the way a server meets it: `requests` of them, the longest of `longest` tokens (new ones
included), the others down to longest/spread, spread evenly over the logarithm; the first `chunked` bring up to `chunk` tokens in
this step, the others one token each, the last `idle` none and hold none.  `batch` seeds these lengths: they are the case's own,
while every value, table and permutation comes from prepare's seed.

The cache: codes of 8 bits (`kind` int8 or e4m3), K as [blocks][kv heads][block][dim], V transposed as
[blocks][kv heads][dim][block], one fp32 scale per block and kv head for each.  The codes and the scales are the state of the
cache, so they are returned as they are held.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TOP = {"int8": 127.0, "e4m3": 448.0}
DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


# ---- cases -------------------------------------------------------------------------------------------------------------

def _case(op, requests, longest, spread=1, chunk=1, chunked=0, idle=0, batch=1, block=64, **more):
    return dict(op=op, requests=requests, longest=longest, spread=spread, chunk=chunk, chunked=chunked, idle=idle, batch=batch,
                block=block, **more)


def _heads(n_q, n_kv, dim):
    return dict(n_q=n_q, n_kv=n_kv, dim=dim)


LAYER = _heads(20, 5, 128)      # the 2B-style layer: 20 query heads over 5 key/value heads of 128


def listed():
    def named(name, case):
        return dict(case, name=name)
    return [
        # the allocator in a small server's decode step: time to the answer is all there is
        named("tables_decode_8", _case("tables", 8, 4096, 8)),
        # a large server's step: decode, prompts that come in whole, requests that end, small blocks
        named("tables_mixed_512", _case("tables", 512, 8192, 64, 1024, 32, 8, block=16)),
        # one generated token of one sequence, one layer's K and V
        named("append_one", _case("append", 1, 1500, kind="int8", source="f32", **LAYER)),
        # a decode step of 64 sequences
        named("append_decode_64", _case("append", 64, 8192, 32, kind="e4m3", source="f32", **dict(LAYER, block=32))),
        # a prompt of the model's own context length
        named("append_prompt_4096", _case("append", 1, 4096, 1, 4096, 1, kind="int8", source="f32", **LAYER)),
        # several ragged prompts at once over smaller heads, bf16 projections
        named("append_prompts_ragged", _case("append", 9, 5001, 8, 5001, 9, kind="e4m3", source="bf16", **dict(_heads(32, 8, 64), block=16))),
        # one generated token of one sequence over a full context: latency
        named("attend_one_4096", _case("attend", 1, 4096, kind="int8", window=0, **LAYER)),
        # a decode step of 64 sequences of all lengths: the stream of the cache
        named("attend_decode_64", _case("attend", 64, 8192, 16, idle=1, kind="int8", window=0, **LAYER)),
        # two very long contexts: few rows, a long axis
        named("attend_long_2", _case("attend", 2, 131071, 2, kind="e4m3", window=0, **dict(_heads(32, 8, 128), block=128))),
        # a few proposed tokens checked at once, sliding window, small heads and blocks
        named("attend_verify_16", _case("attend", 16, 6000, 8, 4, 16, kind="e4m3", window=2000, **dict(_heads(24, 8, 64), block=16))),
        # prompt processing: every token of the context attends
        named("attend_prompt_4096", _case("attend", 1, 4096, 1, 4096, 1, kind="int8", window=0, **LAYER)),
        # chunks of prompts beside decode steps, ragged
        named("attend_mixed_16", _case("attend", 16, 8000, 16, 512, 3, kind="e4m3", window=0, **dict(LAYER, block=32))),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tables", "append", "append", "attend", "attend", "attend"])
    block, batch = rng.choice([16, 32, 64, 128]), rng.randrange(1, 1 << 20)
    if op == "tables":
        requests = _log(rng, 1, 512)
        return _case(op, requests, _log(rng, 64, 16384), _log(rng, 1, 64), _log(rng, 1, 1024), rng.randrange(0, min(32, requests) + 1),
                     rng.randrange(0, requests // 8 + 1), batch, block)
    heads = _heads(*rng.choice([(20, 5, 128), (32, 8, 128), (8, 8, 128), (16, 1, 128), (32, 8, 64), (24, 8, 64), (12, 12, 64)]))
    kind = rng.choice(["int8", "e4m3"])
    if op == "append":
        source = rng.choice(["f32", "bf16"])
        if rng.random() < 0.5:
            return _case(op, _log(rng, 1, 64), _log(rng, 1, 8192), _log(rng, 1, 32), 1, 0, 0, batch, block, kind=kind, source=source, **heads)
        requests = _log(rng, 1, 9)
        longest = _log(rng, 64, 20000 // requests)
        return _case(op, requests, longest, _log(rng, 1, 8), _log(rng, 16, longest), requests, 0, batch, block, kind=kind, source=source, **heads)
    window = rng.choice([0, 0, _log(rng, 100, 4000)])
    what = rng.choice(["decode", "long", "verify", "prompt", "mixed"])
    more = dict(kind=kind, window=window, **heads)
    if what == "decode":
        requests = _log(rng, 1, 64)
        return _case(op, requests, _log(rng, 1, 8192), _log(rng, 1, 32), 1, 0, min(requests // 4, rng.randrange(0, 3)), batch, block, **more)
    if what == "long":
        return _case(op, rng.choice([1, 2]), _log(rng, 16384, 131071), 2, 1, 0, 0, batch, block, **more)
    if what == "verify":
        requests = _log(rng, 1, 32)
        return _case(op, requests, _log(rng, 64, 8192), _log(rng, 1, 16), rng.randrange(2, 9), requests, 0, batch, block, **more)
    if what == "prompt":
        requests = rng.choice([1, 1, 2, 3])
        longest = _log(rng, 32, 4096 // requests)
        return _case(op, requests, longest, 2, longest, requests, 0, batch, block, **more)
    requests = _log(rng, 2, 16)
    return _case(op, requests, _log(rng, 1024, 8000), _log(rng, 1, 16), _log(rng, 16, 512), min(3, requests), 0, batch, block, **more)


def _lengths(case):
    """(tokens in all, new ones among them) of each request."""
    rng, B = random.Random(case["batch"]), case["requests"]
    total, new = [], []
    for b in range(B):
        n = case["longest"] if b == 0 else max(1, int(case["longest"] * case["spread"] ** -rng.random()))
        n = 0 if b >= B - case["idle"] else n
        total.append(n)
        new.append(min(n, case["chunk"] if b < case["chunked"] else 1))
    return total, new


def _blocks(n, block):
    return -(-n // block)


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _paged(case, total, gen, spare):
    """A table of the requests' blocks in a random order over a pool with `spare` blocks more, the last of which nobody has."""
    block = case["block"]
    counts = [_blocks(n, block) for n in total]
    width, used = max(1, max(counts)), sum(counts)
    order = torch.randperm(used + spare, generator=gen, device=DEV).to(torch.int32)
    c = torch.tensor(counts, device=DEV)
    first = (c.cumsum(0) - c)[:, None]
    col = torch.arange(width, device=DEV)[None]
    table = torch.where(col < c[:, None], order[(first + col).clamp(max=used + spare - 1)], -1)
    return table.to(torch.int32).contiguous(), order, used, used + spare + 1


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _normal(gen, *shape, dtype=torch.float32):
    """Values as projections give them: N(0, 1) with one channel in 32 four times as large."""
    x = torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)
    x[..., 5::32] *= 4
    return x.to(dtype)


def _encode(x, kind, dims):
    """Codes and scales of x, one scale over `dims`."""
    scale = x.abs().amax(dims, keepdim=True).clamp(min=1e-5) / TOP[kind]
    y = (x / scale).clamp(-TOP[kind], TOP[kind])
    return (y.round() if kind == "int8" else y).to(DTYPE[kind]), scale


def _cache(case, n_blocks, gen):
    """A cache that earlier steps have filled."""
    H, bs, D, kind = case["n_kv"], case["block"], case["dim"], case["kind"]
    c = {"k": torch.empty(n_blocks, H, bs, D, dtype=DTYPE[kind], device=DEV), "v": torch.empty(n_blocks, H, D, bs, dtype=DTYPE[kind], device=DEV),
         "k_scale": torch.empty(n_blocks, H, device=DEV), "v_scale": torch.empty(n_blocks, H, device=DEV)}
    step = max(1, (1 << 26) // (H * bs * D))
    for i in range(0, n_blocks, step):
        n = min(step, n_blocks - i)
        for name in "kv":
            x, s = _encode(_normal(gen, n, H, bs, D), kind, (2, 3))
            c[name][i:i + n] = x if name == "k" else x.view(torch.uint8).transpose(2, 3).contiguous().view(DTYPE[kind])
            c[name + "_scale"][i:i + n] = s[:, :, 0, 0]
    return c


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    total, new = _lengths(case)
    B, bs = case["requests"], case["block"]
    s = {"case": case, "op": case["op"], "block": bs}
    if case["op"] == "tables":
        # one request in nine ends; the pool has room for most of the demand, so that a full batch is refused now and then
        old = [t - n for t, n in zip(total, new)]
        ends = [b % 9 == 7 for b in range(B)]
        demand = sum(_blocks(t, bs) - _blocks(o, bs) for t, o, e in zip(total, old, ends) if not e)
        table, order, used, n_blocks = _paged(case, old, gen, demand + 16)
        width = max(_blocks(t, bs) for t in total)
        s["table"] = torch.cat([table, torch.full((B, max(0, width - table.shape[1]) + 1), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
        s["free_list"] = torch.cat([order[used:], torch.full((used,), -1, dtype=torch.int32, device=DEV)])
        s["free_count"] = _ints([demand + 16 if seed % 4 else (demand + 16) // 2])
        s["seq_len"] = _ints(old)
        s["new_len"] = _ints([-1 if e else n for n, e in zip(new, ends)])
        s["rows"] = sum(new) + 7                       # rows of the batch: a few are padding
        return s
    H, n_q, D = case["n_kv"], case["n_q"], case["dim"]
    table, order, used, n_blocks = _paged(case, total, gen, 16)
    s.update(_cache(case, n_blocks, gen))
    s.update(kind=case["kind"], n_q=n_q, table=table, seq_len=_ints(total))
    T = sum(new)
    n = torch.tensor(new, device=DEV)
    s["q_start"] = torch.cat([n.new_zeros(1), n.cumsum(0)]).to(torch.int32)
    if case["op"] == "append":
        req = torch.repeat_interleave(torch.arange(B, device=DEV), n, output_size=T)
        pos = torch.arange(T, device=DEV) - s["q_start"][req] + s["seq_len"][req] - n[req]
        s["positions"] = pos.to(torch.int32)
        s["slots"] = (table[req, pos // bs] * bs + pos % bs).to(torch.int32)
        angle = torch.arange(case["longest"], device=DEV, dtype=torch.float64)[:, None] * \
            500000.0 ** (-torch.arange(D // 2, device=DEV, dtype=torch.float64) * 2 / D)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["qkv"] = _normal(gen, T, (n_q + 2 * H) * D, dtype=torch.float32 if case["source"] == "f32" else torch.bfloat16)
        s["runs"] = 2 * B + T // bs
    else:
        s["q"] = _normal(gen, T, n_q, D, dtype=torch.bfloat16)
        s["max_q"], s["max_len"], s["window"] = max(new), max(total), case["window"]
        s["softmax_scale"] = D ** -0.5
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------------

def _tables(s):
    """Ended requests give their blocks back, the others take what they need from the top of the stack, in their order."""
    bs, T, table = s["block"], s["rows"], s["table"]
    B, width = table.shape
    old, new, cap = s["seq_len"].long().clamp(0, width * bs), s["new_len"].long(), s["free_list"].numel()
    ended = new < 0
    n = new.clamp(min=0)
    have, need = (old + bs - 1) // bs, (old + n + bs - 1) // bs
    col = torch.arange(width, device=DEV)[None]
    back = torch.where(ended, have, 0)
    at = s["free_count"].long() + (back.cumsum(0) - back)[:, None] + col
    free = torch.cat([s["free_list"], s["free_list"].new_zeros(1)])
    free[torch.where((col < back[:, None]) & (at < cap), at, cap)] = table
    there = (s["free_count"].long() + back.sum()).clamp(max=cap)
    lost = (ended & (s["free_count"].long() + back.cumsum(0) > cap)).sum()
    end = n.cumsum(0)
    fits = ~ended & (need <= width) & (end <= T)
    want = torch.where(fits, need - have, 0)
    upto = want.cumsum(0)
    ok = fits & ((want == 0) | (upto <= there))
    j = col - have[:, None]
    mine = ok[:, None] & (j >= 0) & (j < want[:, None])
    table = torch.where(mine, free[(there - 1 - (upto - want)[:, None] - j).clamp(0, cap)], table)
    start = torch.where(ok, old, -1)
    q_start = torch.cat([end.new_zeros(1), end.clamp(max=T)])
    t = torch.arange(T, device=DEV)
    req = torch.searchsorted(q_start[1:].contiguous(), t, right=True).clamp(max=B - 1)
    live = (t < q_start[B]) & (start[req] >= 0)
    pos = torch.where(live, start[req] + t - q_start[req], 0)
    slot = torch.where(live, table[req, (pos // bs).clamp(max=width - 1)].long() * bs + pos % bs, -1)
    return {"table": table, "free_list": free[:cap], "free_count": (there - torch.where(ok, upto, 0).amax()).to(torch.int32).reshape(1),
            "seq_len": torch.where(ended, 0, torch.where(ok, old + n, old)).to(torch.int32), "start": start.to(torch.int32),
            "q_start": q_start.to(torch.int32), "positions": pos.to(torch.int32), "slots": slot.to(torch.int32),
            "bad": ((~ended & ~ok).sum() + lost).to(torch.int32).reshape(1)}


def _append(s):
    """Rotary, then codes: a block's scale is that of its largest value so far, and what it holds moves to a scale that grew."""
    kind, bs, top = s["kind"], s["block"], TOP[s["kind"]]
    n_blocks, H = s["k_scale"].shape
    T, D, n_q = s["qkv"].shape[0], s["k"].shape[3], s["n_q"]
    x = s["qkv"].float().view(T, n_q + 2 * H, D)
    cos, sin = s["cos"][s["positions"].long()][:, None], s["sin"][s["positions"].long()][:, None]
    a, b = x[:, :n_q + H, :D // 2], x[:, :n_q + H, D // 2:]
    turned = torch.cat([a * cos - b * sin, b * cos + a * sin], 2)
    # runs of tokens of the same block; a place without a run works on the last block, which nobody has, and leaves it as it is
    blk, off = s["slots"].long() // bs, s["slots"].long() % bs
    lead = torch.cat([blk.new_ones(1, dtype=torch.bool), blk[1:] != blk[:-1]])
    first = torch.argsort((~lead).to(torch.int8), stable=True)[:s["runs"]]
    place, begun, tok = torch.where(lead[first], blk[first], n_blocks - 1), torch.where(lead[first], off[first], 0), torch.arange(bs, device=DEV)
    kept = tok[None] < begun[:, None]
    out = {"q": turned[:, :n_q].to(torch.bfloat16).reshape(T, n_q * D)}
    for name, y in (("k", turned[:, n_q:]), ("v", x[:, n_q + H:])):
        scale, codes = s[name + "_scale"], s[name]
        most = y.abs().amax(2)
        g = torch.zeros(n_blocks, H, device=DEV).scatter_reduce_(0, blk[:, None].expand(T, H), most, "amax")[place]
        old = scale[place]
        now = torch.where(lead[first][:, None], g.clamp(min=1e-5) / top, old)
        now = torch.where((begun > 0)[:, None], torch.maximum(now, old), now)
        scale[place] = now
        ratio = (old / now)[:, :, None, None]
        held = codes[place].float()
        moved = (held * ratio).round() if kind == "int8" else held * ratio
        mask = kept[:, None, :, None] if name == "k" else kept[:, None, None, :]
        codes.view(torch.uint8)[place] = torch.where(mask, moved, held).to(codes.dtype).view(torch.uint8)
        z = (y * (1.0 / scale[blk])[:, :, None]).clamp(-top, top)
        z = (z.round() if kind == "int8" else z).to(codes.dtype).view(torch.uint8)
        if name == "k":
            codes.view(torch.uint8)[blk, :, off] = z
        else:
            codes.view(torch.uint8)[blk, :, :, off] = z
        out[name], out[name + "_scale"] = codes, scale
    return out


def _attend(s):
    """Softmax over the cached tokens up to a query's own position (the last ones of its request are the queries)."""
    table, bs = s["table"].long(), s["block"]
    B, width = table.shape
    n_blocks, H, _, D = s["k"].shape
    T, n_q, _ = s["q"].shape
    G, L, most = n_q // H, width * bs, s["max_q"]
    page = table.clamp(0, n_blocks - 1)
    there = ((table >= 0) & (table < n_blocks))[:, :, None].expand(B, width, bs).reshape(B, L)
    k = s["k"][page].float() * s["k_scale"][page][..., None, None]
    k = k.permute(0, 2, 4, 1, 3).reshape(B, H, D, L)
    v = s["v"][page].float() * s["v_scale"][page][..., None, None]
    v = v.permute(0, 2, 1, 4, 3).reshape(B, H, L, D)
    first, count = s["q_start"][:-1].long(), (s["q_start"][1:] - s["q_start"][:-1]).long()
    i = torch.arange(most, device=DEV)
    q = s["q"][(first[:, None] + i).clamp(max=T - 1)].float().view(B, most, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, most * G, D)
    pos = (s["seq_len"].long() - count)[:, None] + i                       # [B][most]
    j = torch.arange(L, device=DEV)
    seen = (j <= pos[:, :, None]) & there[:, None]
    if s["window"]:
        seen &= j > pos[:, :, None] - s["window"]
    seen = seen[:, None, :, None].expand(B, 1, most, G, L).reshape(B, 1, most * G, L)
    x = torch.matmul(q, k) * s["softmax_scale"]
    x.masked_fill_(~seen, -math.inf)
    x -= x.amax(3, keepdim=True).clamp(min=-3e38)
    x.exp_()
    o = torch.matmul(x, v) / x.sum(3, keepdim=True).clamp(min=1e-38)
    o = o.view(B, H, most, G, D).permute(0, 2, 1, 3, 4).reshape(B, most, n_q * D)
    t = torch.arange(T, device=DEV)
    req = torch.searchsorted(s["q_start"][1:].long().contiguous(), t, right=True).clamp(max=B - 1)
    return o[req, t - first[req]].to(torch.bfloat16)


# ---- one pass ----------------------------------------------------------------------------------------------------------

def _handle(s):
    """What a serving program keeps of a batch: the descriptor over its own buffers."""
    from paper_2504_12285_amd import binding as bl
    if s["op"] == "tables":
        return bl.KVTables(s["seq_len"], s["new_len"], s["table"], s["free_list"], s["free_count"], s["block"], s["rows"])
    cache = bl.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    if s["op"] == "append":
        return bl.KVAppend(cache, s["qkv"], s["n_q"], s["slots"], s["positions"], s["cos"], s["sin"])
    return bl.KVAttention(cache, s["q"], s["q_start"], s["seq_len"], s["table"], max_q=s["max_q"], max_len=s["max_len"],
                          softmax_scale=s["softmax_scale"], window=s["window"])


def _own(s):
    h = s.get("handle")
    if h is None:
        h = s["handle"] = _handle(s)
    h.run()
    if s["op"] == "tables":
        return {"table": h.table, "free_list": h.free_list, "free_count": h.free_count_out, "seq_len": h.seq_len_out, "start": h.start,
                "q_start": h.q_start, "positions": h.positions, "slots": h.slots, "bad": h.bad}
    if s["op"] == "append":
        return {"q": h.q, "k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    return {"out": h.out}


def run(state):
    if own:
        return _own(state)
    if state["op"] == "tables":
        return _tables(state)
    return _append(state) if state["op"] == "append" else {"out": _attend(state)}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    total, new = _lengths(case)
    T, B, bs = sum(new), case["requests"], case["block"]
    if case["op"] == "tables":
        fresh = sum(_blocks(t, bs) - _blocks(t - n, bs) for t, n in zip(total, new))
        return {"bytes": 8 * B + 16 * B + 8 * T + 12 * fresh, "flops": 0}
    H, n_q, D = case["n_kv"], case["n_q"], case["dim"]
    if case["op"] == "append":
        row = (n_q + 2 * H) * D * (4 if case["source"] == "f32" else 2) + n_q * D * 2 + 2 * H * D + 4 * D + 8
        runs = sum(_blocks(t, bs) - (t - n) // bs for t, n in zip(total, new))
        return {"bytes": T * row + runs * H * 8, "flops": 0}
    w = case["window"] or 1 << 40
    read = sum(min(t, n + w - 1) for t, n in zip(total, new))
    pairs = 0
    for t, n in zip(total, new):
        full = max(0, min(n, t - w))                       # queries whose window is whole
        pairs += full * w if full else 0
        pairs += sum(range(t - n + 1, t - full + 1)) if n - full else 0
    return {"bytes": read * H * D * 2 + sum(_blocks(t, bs) for t in total) * (8 * H + 4) + T * n_q * D * 4, "flops": 4 * pairs * n_q * D}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "tables":
        return None
    s = prepare(case, seed)
    total, new = _lengths(case)
    n_q, H, D, bs = case["n_q"], case["n_kv"], case["dim"], case["block"]
    starts = s["q_start"].tolist()
    if case["op"] == "append":
        T = starts[-1]
        x = s["qkv"].double().view(T, n_q + 2 * H, D)
        z = torch.complex(x[..., :D // 2], x[..., D // 2:])
        p = s["positions"].long()
        z = z * torch.complex(s["cos"][p].double(), s["sin"][p].double())[:, None]
        r = torch.cat([z.real, z.imag], 2)
        r[:, n_q + H:] = x[:, n_q + H:]
        scales = {"k_scale": s["k_scale"].double(), "v_scale": s["v_scale"].double()}
        for b, (t, n) in enumerate(zip(total, new)):
            pages = s["table"][b].tolist()
            at = t - n
            while at < t:
                end = min(t, (at // bs + 1) * bs)
                rows = r[starts[b] + at - (t - n):starts[b] + end - (t - n)]
                for name, y in (("k_scale", rows[:, n_q:n_q + H]), ("v_scale", rows[:, n_q + H:])):
                    g = y.abs().amax((0, 2)).clamp(min=1e-5) / TOP[case["kind"]]
                    held = scales[name][pages[at // bs]]
                    scales[name][pages[at // bs]] = torch.maximum(g, held) if at % bs else g
                at = end
        return {"q": r[:, :n_q].reshape(T, n_q * D), "k": None, "v": None, **scales}
    out = torch.zeros(starts[-1], n_q, D, dtype=torch.float64, device=DEV)
    for b, (t, n) in enumerate(zip(total, new)):
        if n == 0:
            continue
        pages = s["table"][b, :_blocks(t, bs)].long()
        k = (s["k"][pages].double() * s["k_scale"][pages].double()[..., None, None]).transpose(0, 1).reshape(H, -1, D)[:, :t]
        v = (s["v"][pages].double() * s["v_scale"][pages].double()[..., None, None]).permute(1, 2, 0, 3).reshape(H, D, -1)[:, :, :t]
        for lo in range(0, n, 1024):
            hi = min(n, lo + 1024)
            at = torch.arange(t - n + lo, t - n + hi, device=DEV)[:, None]
            j = torch.arange(t, device=DEV)[None]
            hide = (j > at) | ((j <= at - case["window"]) if case["window"] else (j < 0))
            for h in range(n_q):
                g = h // (n_q // H)
                x = s["q"][starts[b] + lo:starts[b] + hi, h].double() @ k[g].T * s["softmax_scale"]
                p = torch.softmax(x.masked_fill(hide, -math.inf), 1)
                out[starts[b] + lo:starts[b] + hi, h] = p @ v[g].T
    return {"out": out.reshape(-1, n_q * D)}
