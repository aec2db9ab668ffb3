"""Performance cases of the serving operators: the 8-bit key/value cache and what works on it, through
paper_2511_04002_amd.cache.Cache.

A case names an operator, head counts, the cache's block size, how many requests there are and how long, and a
number format.  `listed` holds the kinds of use, `draw` gives more from the same ranges, `prepare` makes what a
program has in hand before the call, `run` is one pass, `work` the bytes and operations that a pass cannot do
without, `exact` the same results in 64 bits.

Where `own` is false, `run` computes the operators from elementary torch operations in 32 bits, rounded once at
the end; where it is true, it calls the library.

Layout of the cache (both forms): keys int8 [blocks, kv heads, block tokens, head dim], values int8 [blocks, kv
heads, head dim, block tokens], one binary32 scale for each block and kv head of either.
"""
import math
import random

import torch

own = False

# Operators:
#   schedule      block tables, slot map and positions from the requests' lengths and their new tokens
#   norm_rotate   RMS norm of each head's query and key, and the position rotation
#   append        new keys and values into the cache; returns the values that the touched blocks then stand for
#   gather        the last tokens of each request out of the cache
#   attend        attention of the new tokens' queries over the cache


def _case(name, op, dtype, q_heads, kv_heads, dim, block, requests, past, new, mix=0, rows="even", causal=True, window=0,
          pairs="halves", rotary=0, norm=True):
    """past, new: the longest request's tokens in the cache before the step, and the most new tokens of a request;
    rows: "even" (all requests the same), "ragged" (each request its own, drawn by the number `mix`)."""
    case = dict(op=op, dtype=dtype, q_heads=q_heads, kv_heads=kv_heads, dim=dim, block=block, requests=requests, past=past,
                new=new, mix=mix, rows=rows, causal=causal, window=window, pairs=pairs, rotary=rotary or dim, norm=norm)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # a generated token each of 512 sequences: where do they go
        _case("schedule_decode", "schedule", "f16", 40, 40, 128, 16, 512, 4096, 1, mix=1, rows="ragged"),
        # 32 prompts of up to 4096 tokens arrive at once
        _case("schedule_prompts", "schedule", "bf16", 64, 8, 128, 16, 32, 0, 4096, mix=2, rows="ragged"),
        # one token of a small model: latency alone
        _case("norm_rotate_token", "norm_rotate", "f16", 12, 12, 64, 16, 1, 127, 1),
        # a long prompt of a large model
        _case("norm_rotate_prompt", "norm_rotate", "bf16", 64, 8, 128, 16, 1, 0, 8192),
        # a token each of 512 sequences (13B-shaped) into blocks that are partly full
        _case("append_decode", "append", "f16", 40, 40, 128, 16, 512, 1024, 1, mix=3, rows="ragged"),
        # prompts of odd lengths (7B-shaped)
        _case("append_prompts", "append", "f16", 32, 32, 128, 32, 5, 333, 2048, mix=4, rows="ragged"),
        # a request's whole cache, to be sent on: one layer of 2048 tokens (7B-shaped), and odd ones of many requests
        _case("gather_request", "gather", "f16", 32, 32, 128, 16, 1, 0, 2048),
        _case("gather_ragged", "gather", "bf16", 64, 8, 128, 64, 37, 0, 4097, mix=5, rows="ragged"),
        # one token of a small model over a short cache: latency alone
        _case("attend_token", "attend", "f16", 12, 12, 64, 16, 1, 127, 1),
        # a token each of 64 sequences of up to 4096 (13B-shaped, a key head for each query head)
        _case("attend_decode", "attend", "f16", 40, 40, 128, 16, 64, 4095, 1, mix=6, rows="ragged"),
        # one very long sequence, eight query heads to a key head: the work is along the cache alone
        _case("attend_long", "attend", "bf16", 64, 8, 128, 16, 1, 131071, 1),
        # prefill of a long prompt (70B-shaped)
        _case("attend_prompt", "attend", "bf16", 64, 8, 128, 16, 1, 0, 8192),
    ]


HEADS = [(12, 12, 64), (20, 20, 64), (32, 32, 128), (40, 40, 128), (32, 8, 128), (40, 8, 128), (64, 8, 128), (28, 4, 128),
         (16, 2, 128), (8, 1, 128), (16, 8, 256), (8, 1, 256)]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))


def draw(rng):
    op = rng.choice(["schedule", "norm_rotate", "append", "gather", "attend", "attend", "attend", "attend"])
    q_heads, kv_heads, dim = rng.choice(HEADS)
    dtype, block = rng.choice(["f16", "bf16"]), rng.choice([16, 16, 32, 64, 128])
    rows = rng.choice(["even", "ragged", "ragged"])
    mix = rng.randrange(1 << 20)
    more = {}
    if op == "schedule":
        requests = int(_log_uniform(rng, 1, 2048))
        new = 1 if rng.random() < 0.5 else int(_log_uniform(rng, 1, max(1, min(8192, 131072 // requests))))
        past = 0 if rng.random() < 0.2 else int(_log_uniform(rng, 1, min(131072, 4194304 // requests)))
    elif op == "norm_rotate":
        requests = int(_log_uniform(rng, 1, 512))
        new = int(_log_uniform(rng, 1, max(1, (8192 * 72 * 128) // ((q_heads + kv_heads) * dim * requests))))
        past = int(_log_uniform(rng, 1, 8192))
        more = dict(pairs=rng.choice(["halves", "neighbours"]), rotary=rng.choice([dim, dim, dim // 2]),
                    norm=rng.random() < 0.75)
    elif op == "append":
        requests = int(_log_uniform(rng, 1, 512))
        most = max(1, (5 * 2048 * 32 * 128) // (kv_heads * dim * requests))
        new = 1 if rng.random() < 0.4 else int(_log_uniform(rng, 1, min(8192, most)))
        past = int(_log_uniform(rng, 1, max(1, min(8192, (1 << 29) // (kv_heads * dim * requests)))))
    elif op == "gather":
        requests = int(_log_uniform(rng, 1, 64))
        new = int(_log_uniform(rng, 1, min(16384, (1 << 27) // (kv_heads * dim * requests))))
        past = rng.choice([0, 0, rng.randrange(1000)])
    else:
        kind = rng.choice(["token", "token", "few", "chunk", "prompt"])
        if kind in ("token", "few"):
            new = 1 if kind == "token" else rng.randint(2, 8)
            requests = int(_log_uniform(rng, 1, 256))
            # elements of the keys, padded to the longest: no more than a listed case has
            past = int(_log_uniform(rng, 1, min(131071, (64 * 4096 * 40 * 128) // (kv_heads * dim * requests))))
        elif kind == "chunk":
            requests, new = rng.randint(1, 8), int(_log_uniform(rng, 9, 1024))
            past = int(_log_uniform(rng, 1, max(1, min(65536, (1 << 31) // (q_heads * new * requests)))))
        else:
            requests = rng.randint(1, 6)
            most = math.isqrt((1 << 31) * 128 // (q_heads * dim * requests))
            new, past = int(_log_uniform(rng, 16, min(8192, most))), 0
        more = dict(causal=rng.random() < 0.85, window=rng.choice([0, 0, 0, int(_log_uniform(rng, 16, 4096))]))
    return _case(None, op, dtype, q_heads, kv_heads, dim, block, requests, past, new, mix=mix, rows=rows, **more)


# ------------------------------------------------------------------ what a case's requests are

def _requests(case):
    """-> (tokens in the cache before the step, new tokens) of each request."""
    n, past, new = case["requests"], case["past"], case["new"]
    if case["rows"] == "even":
        return [past] * n, [new] * n
    rng = random.Random(case["mix"])
    pasts = [rng.randint(past // 4, past) for _ in range(n)]
    news = [rng.randint((new + 3) // 4, new) for _ in range(n)]
    at = rng.randrange(n)
    pasts[at], news[at] = past, new
    return pasts, news


def _blocks(tokens, block):
    return (tokens + block - 1) // block


def _kind(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


class _State:
    pass


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = random.Random(seed)
    s = _State()
    s.op, s.case = case["op"], case
    s.block, s.q_heads, s.kv_heads, s.dim = case["block"], case["q_heads"], case["kv_heads"], case["dim"]
    s.kind = _kind(case)
    pasts, news = _requests(case)
    lengths = [p + n for p, n in zip(pasts, news)]
    s.requests, s.tokens = len(news), sum(news)
    s.max_new, s.max_length = max(news), max(lengths)
    s.starts = _ints(_starts(news))
    s.lengths, s.pasts, s.new = _ints(lengths), _ints(pasts), _ints(news)
    # a pool that has been in use: blocks anywhere in it, a tenth of them free behind the step
    held = [_blocks(n, s.block) for n in lengths]
    s.blocks = sum(held) + sum(held) // 10 + 1
    s.max_blocks = _blocks(s.max_length, s.block)

    def randn(*shape, scale=1.0):
        return (torch.randn(shape, device="cuda", generator=gen) * scale).to(s.kind)

    if own:
        from paper_2511_04002_amd import cache
        s.cache = cache.Cache(s.blocks, s.block, s.q_heads, s.kv_heads, s.dim, case["dtype"], s.max_blocks)
    if s.op == "schedule":
        order = torch.randperm(s.blocks, device="cuda", generator=gen).to(torch.int32)
        before = [_blocks(n, s.block) for n in pasts]
        if s.requests > 4:                       # some requests are done: their blocks go back
            done = random.Random(case["mix"] + 1)
            news = [-1 if p and done.random() < 0.05 else n for p, n in zip(pasts, news)]
            s.new = _ints(news)
            s.tokens = sum(max(n, 0) for n in news)
        s.table = torch.full((s.requests, s.max_blocks), -1, dtype=torch.int32, device="cuda")
        if sum(before):
            row = torch.repeat_interleave(torch.arange(s.requests, device="cuda"), torch.tensor(before, device="cuda"))
            first = torch.tensor(_starts(before)[:-1], device="cuda")
            s.table[row, torch.arange(sum(before), device="cuda") - first[row]] = order[:sum(before)]
        # the ring of free blocks, which has gone round before
        taken, free = rng.randrange(10 * s.blocks), order[sum(before):]
        s.ring = torch.full((s.blocks,), -1, dtype=torch.int32, device="cuda")
        s.ring[(taken + torch.arange(free.numel(), device="cuda")) % s.blocks] = free
        s.counters = torch.tensor([taken, taken + free.numel()], dtype=torch.int64, device="cuda")
        if own:
            s.out = s.cache.new_schedule(s.requests, s.tokens)
        return s
    if s.op == "norm_rotate":
        width = (s.q_heads + 2 * s.kv_heads) * s.dim
        s.qkv = randn(s.tokens, width)           # one projection's output holds queries, keys and values
        s.qkv[:, torch.randperm(width, device="cuda", generator=gen)[:8]] *= 20.0
        s.q = s.qkv[:, :s.q_heads * s.dim].unflatten(1, (s.q_heads, s.dim))
        s.k = s.qkv[:, s.q_heads * s.dim:(s.q_heads + s.kv_heads) * s.dim].unflatten(1, (s.kv_heads, s.dim))
        s.q_weight = s.k_weight = None
        if case["norm"]:
            s.q_weight, s.k_weight = (1 + randn(s.dim, scale=0.2).float()).to(s.kind), (1 + randn(s.dim, scale=0.2).float()).to(s.kind)
        half = case["rotary"] // 2
        rate = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        angle = torch.arange(s.max_length, device="cuda", dtype=torch.float64)[:, None] * rate
        s.angles = torch.cat((angle.cos(), angle.sin()), 1).float()
        s.eps, s.pairs = 1e-6, case["pairs"]
        s.positions = _ints([p + i for p, n in zip(pasts, news) for i in range(n)])
        s.q_out = torch.empty((s.tokens, s.q_heads, s.dim), dtype=s.kind, device="cuda")
        s.k_out = torch.empty((s.tokens, s.kv_heads, s.dim), dtype=s.kind, device="cuda")
        return s
    # the cache: any block may be in use by any request, places behind a request's end hold what was there before
    s.k = torch.empty((s.blocks, s.kv_heads, s.block, s.dim), dtype=torch.int8, device="cuda")
    s.v = torch.empty((s.blocks, s.kv_heads, s.dim, s.block), dtype=torch.int8, device="cuda")
    s.v_scale, s.k_scale = (torch.exp(0.3 * torch.randn((s.blocks, s.kv_heads), device="cuda", generator=gen)) / 36 for _ in range(2))
    per = max(1, (1 << 27) // (s.kv_heads * s.block * s.dim))
    for at in range(0, s.blocks, per):
        for t in (s.k, s.v):
            part = t[at:at + per]
            part.copy_(torch.randn(part.shape, device="cuda", generator=gen).mul_(36).clamp_(-127, 127).round_())
    order = torch.randperm(s.blocks, device="cuda", generator=gen).to(torch.int32)
    s.table = torch.full((s.requests, s.max_blocks), -1, dtype=torch.int32, device="cuda")
    row = torch.repeat_interleave(torch.arange(s.requests, device="cuda"), torch.tensor(held, device="cuda"))
    first = torch.tensor(_starts(held)[:-1], device="cuda")
    s.table[row, torch.arange(sum(held), device="cuda") - first[row]] = order[:sum(held)]
    if own:
        s.memory = s.cache.wrap(s.k, s.v, s.k_scale, s.v_scale)
    # row of the step -> its request and its position there
    s.row = torch.repeat_interleave(torch.arange(s.requests, device="cuda"), s.new.long())
    s.at = torch.arange(s.tokens, device="cuda") - s.starts.long()[s.row] + s.pasts.long()[s.row]
    if s.op == "append":
        s.slots = (s.table[s.row, s.at // s.block].long() * s.block + s.at % s.block).to(torch.int32)
        s.new_k = randn(s.tokens, s.kv_heads, s.dim)
        s.new_v = randn(s.tokens, s.kv_heads, s.dim, scale=0.6)
        s.new_k[:, :, torch.randperm(s.dim, device="cuda", generator=gen)[:2]] *= 8.0
        # what the step touches: from the first token of the first block that it writes to
        firsts = [p // s.block * s.block for p in pasts]
        counts = [n - f for n, f in zip(lengths, firsts)]
        s.tokens = sum(counts)
        s.starts = _ints(_starts(counts))
        s.row = torch.repeat_interleave(torch.arange(s.requests, device="cuda"), torch.tensor(counts, device="cuda"))
        s.at = torch.arange(s.tokens, device="cuda") - s.starts.long()[s.row] + torch.tensor(firsts, device="cuda")[s.row]
    if s.op in ("append", "gather"):
        s.k_out, s.v_out = (torch.empty((s.tokens, s.kv_heads, s.dim), dtype=s.kind, device="cuda") for _ in range(2))
        return s
    s.q = randn(s.tokens, s.q_heads, s.dim, scale=1.5)
    s.scale, s.causal, s.window = s.dim ** -0.5, case["causal"], case["window"]
    s.out = torch.empty((s.tokens, s.q_heads, s.dim), dtype=s.kind, device="cuda")
    s.lse = torch.empty((s.tokens, s.q_heads), dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return (_library if own else _plain)(s)


def _library(s):
    if s.op == "schedule":
        s.cache.schedule(s.new, s.pasts, s.table, s.ring, s.counters, s.out)
        o = s.out
        return {"table": s.table, "ring": s.ring, "lengths": o.lengths, "counters": o.counters, "starts": o.starts,
                "positions": o.positions, "slots": o.slots}
    if s.op == "norm_rotate":
        s.cache.norm_rotate(s.q, s.k, s.positions, s.angles, s.q_weight, s.k_weight, s.eps, s.pairs, s.q_out, s.k_out)
        return {"q": s.q_out, "k": s.k_out}
    if s.op == "append":
        s.cache.append(s.memory, s.new_k, s.new_v, s.slots)
    if s.op in ("append", "gather"):
        s.cache.gather(s.memory, s.table, s.starts, s.lengths, s.k_out, s.v_out)
        return {"k": s.k_out, "v": s.v_out}
    s.cache.attend(s.memory, s.q, s.table, s.starts, s.lengths, s.max_new, s.max_length, s.scale, s.causal, s.window, s.out, s.lse)
    return {"out": s.out, "lse": s.lse}


def _plain(s):
    return {"schedule": _plain_schedule, "norm_rotate": _plain_norm_rotate, "append": _plain_append, "gather": _plain_gather,
            "attend": _plain_attend}[s.op](s)


def _plain_schedule(s):
    device, block = s.new.device, s.block
    new, past = s.new.long(), s.pasts.long()
    grow, gone = new.clamp(min=0), new < 0
    lengths = torch.where(gone, 0, past + grow)
    held = (past + block - 1) // block
    more = torch.where(gone, 0, (lengths + block - 1) // block - held)
    back = torch.where(gone, held, 0)
    wanted, returned = more.sum(), back.sum()
    # new blocks, in the order of the requests
    row = torch.repeat_interleave(torch.arange(s.requests, device=device), more)
    nth = torch.arange(row.numel(), device=device)
    column = held[row] + nth - (more.cumsum(0) - more)[row]
    s.table[row, column] = s.ring[(s.counters[0] + nth) % s.blocks]
    # blocks of the requests that are done, in the order of the requests and of their tokens
    row = torch.repeat_interleave(torch.arange(s.requests, device=device), back)
    nth = torch.arange(row.numel(), device=device)
    s.ring[(s.counters[1] + nth) % s.blocks] = s.table[row, nth - (back.cumsum(0) - back)[row]]
    starts = torch.cat((torch.zeros(1, dtype=torch.int64, device=device), grow.cumsum(0)))
    row = torch.repeat_interleave(torch.arange(s.requests, device=device), grow)
    at = torch.arange(row.numel(), device=device) - starts[row] + past[row]
    slots = s.table[row, at // block].long() * block + at % block
    return {"table": s.table, "ring": s.ring, "lengths": lengths.int(), "counters": s.counters + torch.stack((wanted, returned)),
            "starts": starts.int(), "positions": at.int(), "slots": slots.int()}


def _rotated(x, weight, s, angles):
    x = x.to(angles.dtype)
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s.eps) * weight.to(angles.dtype)
    rotary = angles.shape[1]
    c, d = angles[s.positions.long()][:, None, :].split(rotary // 2, -1)
    turn, rest = x[..., :rotary], x[..., rotary:]
    if s.pairs == "halves":
        a, b = turn.split(rotary // 2, -1)
        return torch.cat((a * c - b * d, b * c + a * d, rest), -1)
    a, b = turn[..., 0::2], turn[..., 1::2]
    return torch.cat((torch.stack((a * c - b * d, b * c + a * d), -1).flatten(-2), rest), -1)


def _plain_norm_rotate(s):
    return {"q": _rotated(s.q, s.q_weight, s, s.angles).to(s.kind), "k": _rotated(s.k, s.k_weight, s, s.angles).to(s.kind)}


def _read(codes, scale, block, place, kind):
    """[rows, kv heads, dim] of the cache; codes [blocks, kv heads, block tokens, dim]."""
    return (codes[block, :, place].float() * scale[block][:, :, None]).to(kind)


def _plain_gather(s):
    block, place = s.table[s.row, s.at // s.block].long(), s.at % s.block
    return {"k": _read(s.k, s.k_scale, block, place, s.kind), "v": _read(s.v.transpose(2, 3), s.v_scale, block, place, s.kind)}


def _store(codes, scale, x, slots, size):
    """x [rows, kv heads, dim] into codes [blocks, kv heads, block tokens, dim] and scale [blocks, kv heads]."""
    x, slots = x.float(), slots.long()
    block, place = slots // size, slots % size
    # a block that a row begins is new: what it held counts for nothing
    old = scale.clone()
    old[block[place == 0]] = 0.0
    most = (x.abs().amax(-1) / 127.0)
    most = torch.where(most < 2.0 ** -126, 0.0, most)
    now = old.scatter_reduce(0, block[:, None].expand_as(most), most, "amax")
    touched = torch.unique(block)
    factor = torch.where(now[touched] > 0, old[touched] / now[touched], 1.0)
    codes[touched] = torch.round(codes[touched].float() * factor[:, :, None, None]).to(torch.int8)
    scale[touched] = now[touched]
    inverse = torch.where(now > 0, 1.0 / now, 0.0)
    codes[block, :, place] = torch.round(x * inverse[block][:, :, None]).clamp(-127, 127).to(torch.int8)


def _plain_append(s):
    _store(s.k, s.k_scale, s.new_k, s.slots, s.block)
    _store(s.v.transpose(2, 3), s.v_scale, s.new_v, s.slots, s.block)
    return _plain_gather(s)


def _plain_attend(s):
    group, size = s.q_heads // s.kv_heads, s.block
    # every request padded to the longest: keys and values [requests, kv heads, tokens, dim]
    blocks = (s.max_length + size - 1) // size
    table = s.table[:, :blocks].long().clamp(min=0)
    k = s.k[table].float() * s.k_scale[table][..., None, None]
    k = k.permute(0, 2, 1, 3, 4).reshape(s.requests, s.kv_heads, blocks * size, s.dim)
    v = s.v[table].float() * s.v_scale[table][..., None, None]
    v = v.permute(0, 2, 1, 4, 3).reshape(s.requests, s.kv_heads, blocks * size, s.dim)
    nth = torch.arange(s.tokens, device=s.q.device) - s.starts.long()[s.row]
    q = torch.zeros((s.requests, s.max_new, s.q_heads, s.dim), device=s.q.device)
    q[s.row, nth] = s.q.float()
    q = q.reshape(s.requests, s.max_new, s.kv_heads, group, s.dim).permute(0, 2, 3, 1, 4).reshape(
        s.requests, s.kv_heads, group * s.max_new, s.dim)
    score = torch.matmul(q, k.transpose(2, 3)).mul_(s.scale).view(s.requests, s.kv_heads, group, s.max_new, blocks * size)
    token = torch.arange(blocks * size, device=s.q.device)
    length = s.lengths.long()[:, None, None]
    at = length - s.new.long()[:, None, None] + torch.arange(s.max_new, device=s.q.device)[:, None]
    seen = token < length
    if s.causal:
        seen = seen & (token <= at)
    if s.window:
        seen = seen & (token > at - s.window)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    most = score.amax(-1, keepdim=True)
    score.sub_(torch.where(most == -math.inf, 0.0, most)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(s.requests, s.kv_heads, group * s.max_new, blocks * size), v)
    out = out.view(s.requests, s.kv_heads, group, s.max_new, s.dim) / torch.where(total > 0, total, 1.0)
    out = out.permute(0, 3, 1, 2, 4).reshape(s.requests, s.max_new, s.q_heads, s.dim)[s.row, nth]
    lse = (most + total.log()).permute(0, 3, 1, 2, 4).reshape(s.requests, s.max_new, s.q_heads)[s.row, nth]
    return {"out": out.to(s.kind), "lse": lse}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    pasts, news = _requests(case)
    heads, dim, size = case["kv_heads"], case["dim"], case["block"]
    tokens = sum(news)
    if case["op"] == "schedule":
        more = sum(_blocks(p + n, size) - _blocks(p, size) for p, n in zip(pasts, news))
        return {"bytes": 16 * len(news) + 8 * tokens + 8 * more + 36, "flops": 0}
    if case["op"] == "norm_rotate":
        places = len(set().union(*(range(p, p + n) for p, n in zip(pasts, news))))
        return {"bytes": 4 * tokens * (case["q_heads"] + heads) * dim + 4 * tokens + 4 * places * case["rotary"], "flops": 0}
    if case["op"] == "gather":
        blocks = sum(_blocks(p + n, size) - p // size for p, n in zip(pasts, news))
        return {"bytes": 6 * tokens * heads * dim + 8 * blocks * heads, "flops": 0}
    if case["op"] == "append":
        touched = sum(p + n - p // size * size for p, n in zip(pasts, news))
        blocks = sum(_blocks(p + n, size) - p // size for p, n in zip(pasts, news))
        return {"bytes": 6 * tokens * heads * dim + 4 * tokens + 16 * blocks * heads + 6 * touched * heads * dim, "flops": 0}
    pairs = reach = 0
    for p, n in zip(pasts, news):
        first = lambda at: max(0, at - case["window"] + 1) if case["window"] else 0  # noqa: E731
        last = lambda at: at + 1 if case["causal"] else p + n                        # noqa: E731
        pairs += sum(last(at) - first(at) for at in range(p, p + n))
        reach += p + n - first(p)
    rows = tokens * case["q_heads"]
    return {"bytes": 2 * reach * heads * dim + 8 * heads * reach / size + 4 * rows * dim + 4 * rows,
            "flops": 4 * pairs * case["q_heads"] * dim}


# ------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    if case["op"] == "schedule":
        return None                              # whole numbers
    s = prepare(case, seed)
    if case["op"] == "norm_rotate":
        out = {}
        for name, x, weight in (("q", s.q, s.q_weight), ("k", s.k, s.k_weight)):
            y = x.double()
            if weight is not None:
                y = y / ((y ** 2).sum(-1, keepdim=True) / s.dim + s.eps).sqrt() * weight.double()
            half = case["rotary"] // 2
            turn = torch.complex(s.angles[:, :half].double(), s.angles[:, half:].double())[s.positions.long()][:, None]
            if s.pairs == "halves":
                first, second = slice(0, half), slice(half, 2 * half)
            else:
                first, second = slice(0, 2 * half, 2), slice(1, 2 * half, 2)
            z = torch.complex(y[..., first], y[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            out[name] = y
        return out
    if case["op"] in ("append", "gather"):
        out = {}
        for name, codes, scale in (("k", s.k, s.k_scale.double()), ("v", s.v.transpose(2, 3), s.v_scale.double())):
            codes = codes.double()
            if case["op"] == "append":
                x = (s.new_k if name == "k" else s.new_v).double()
                slots = s.slots.long()
                block, place = slots // s.block, slots % s.block
                before = scale.clone()
                before[block[place == 0]] = 0
                for at in range(s.block):        # one token of a block at a time
                    hit = place == at
                    scale[block[hit]] = torch.maximum(torch.where(torch.tensor(at == 0, device="cuda"), 0, scale[block[hit]]),
                                                      x[hit].abs().amax(-1) / 127)
                ratio = torch.where(scale > 0, before / scale, 1.0)
                codes = (codes * ratio[:, :, None, None]).round()
                codes[block, :, place] = (x / scale[block][:, :, None].clamp(min=1e-300)).round()
            held = s.table[s.row, s.at // s.block].long()
            out[name] = codes[held, :, s.at % s.block] * scale[held][:, :, None]
        return out
    group = s.q_heads // s.kv_heads
    out = torch.zeros((s.tokens, s.q_heads, s.dim), dtype=torch.float64, device="cuda")
    lse = torch.full((s.tokens, s.q_heads), -math.inf, dtype=torch.float64, device="cuda")
    pasts, news = _requests(case)
    starts = _starts(news)
    # a kv head of a request at a time, or of all requests that are one token each a few at a time
    if sum(p + n for p, n in zip(pasts, news)) * s.kv_heads > (1 << 23) and case["new"] > 8:
        return None
    for r, (p, n) in enumerate(zip(pasts, news)):
        held = s.table[r, :_blocks(p + n, s.block)].long()
        token = torch.arange(p + n, device="cuda")
        at = torch.arange(p, p + n, device="cuda")[:, None]
        hidden = torch.zeros((n, p + n), dtype=torch.bool, device="cuda")
        if s.causal:
            hidden |= token > at
        if s.window:
            hidden |= token <= at - s.window
        step = max(1, min(s.kv_heads, (1 << 28) // (group * n * (p + n) + (p + n) * s.dim)))
        for h in range(0, s.kv_heads, step):
            hs = slice(h, min(h + step, s.kv_heads))
            k = s.k[held, hs].double() * s.k_scale[held, hs, None, None].double()
            v = s.v[held, hs].double() * s.v_scale[held, hs, None, None].double()
            k = k.transpose(0, 1).flatten(1, 2)[:, :p + n]
            v = v.permute(1, 0, 3, 2).flatten(1, 2)[:, :p + n]
            rows = slice(starts[r], starts[r + 1])
            q = s.q[rows].double().unflatten(1, (s.kv_heads, group))[:, hs].permute(1, 2, 0, 3)
            weight = (q.flatten(1, 2) @ k.transpose(1, 2)).unflatten(1, (group, n)) * s.scale
            weight = weight.masked_fill(hidden, -math.inf)
            one = weight.logsumexp(-1, keepdim=True)
            weight = (weight - one).exp().nan_to_num(0.0)
            got = (weight.flatten(1, 2) @ v).unflatten(1, (group, n)).permute(2, 0, 1, 3).flatten(1, 2)
            out[rows, hs.start * group:hs.stop * group] = got
            lse[rows, hs.start * group:hs.stop * group] = one[..., 0].permute(2, 0, 1).flatten(1, 2)
    return {"out": out, "lse": lse}
