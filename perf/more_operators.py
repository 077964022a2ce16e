"""Operator cases: a decoder layer's cache of keys and values held in 8 bits, the attention over it, and the tables of its pages.

A served model holds as many tokens as its memory has room for, and reads all of a sequence's tokens for each new one.  Held as whole
numbers of 8 bits with a scale for each block of tokens and head, keys and values take half the room and half the reading.  Kinds of case:

* ``append``: rotary positions on queries and keys; keys and values into the blocks of their sequences.  A block's scale is the smallest
  power of two that lets every value in it be held; a block that a larger value joins is held anew with the larger scale.
* ``attend``: causal attention of new tokens over such a cache: a token a sequence, whole prompts, pieces of prompts, with or without a sliding
  window and sinks, with or without a prefix that all sequences share.  Pages that no row can see any more are not there (-1).
* ``tables``: a step's preparation on the GPU: from the tokens that sequences hold and get, the table of pages (pages that no row will see go
  back, pages for new tokens are taken from those that are free, in order), lengths, first rows, and each row's place, position and sequence.

Heads, head sizes and layer shapes are those of Llama-7B and Llama-13B (32 and 40 heads of 128) and generic grouped ones.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def case(name, op, type="bf16", x_type="bf16", heads=32, kv_heads=32, head_dim=128, page=64, block=16, seqs=1, new=1, len=1024, spread=0,
         window=0, sinks=0, prefix=0, rot=0, pairing="halves"):
    """type: of turned queries and of the attention's queries and results; block: tokens that share a scale."""
    c = dict(op=op, type=type, x_type=x_type, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, block=block, seqs=seqs, new=new,
             len=len, spread=spread, window=window, sinks=sinks, prefix=prefix, rot=rot, pairing=pairing)
    return dict(c, name=name) if name else c


def tables_case(name, seqs=1, page=64, entries=64, new=1, held=1000, spread=0, window=0, sinks=0, prefix=0, idle=0, ended=0, free=200, pad=64):
    """entries: of a sequence's row of the table; idle, ended: every so many sequences gets no token, or is over (0: none); free: pages that are free,
    in percent of those that the step takes; pad: rows are a multiple of this."""
    c = dict(op="tables", seqs=seqs, page=page, entries=entries, new=new, held=held, spread=spread, window=window, sinks=sinks, prefix=prefix,
             idle=idle, ended=ended, free=free, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a generated token of Llama-7B, straight from the products' fp32 results: latency is all
        case("append one token", "append", x_type="f32", len=1000, rot=128),
        # a step of a served batch with grouped heads
        case("append batch of tokens", "append", kv_heads=8, block=32, seqs=96, len=4000, spread=8, rot=128),
        # the prompt of Llama-13B
        case("append long prompt", "append", heads=40, kv_heads=40, page=128, block=64, new=8192, len=8192, rot=128),
        # a generated token of Llama-7B
        case("attend one token", "attend", len=1999),
        # one token over a very long context
        case("attend token, long context", "attend", heads=64, kv_heads=8, page=128, block=128, len=131071),
        # a step of a served batch, contexts of all lengths
        case("attend batch of tokens", "attend", kv_heads=8, page=32, block=32, seqs=64, len=8192, spread=16),
        # pieces of prompts through a window, small heads, odd lengths
        case("attend ragged pieces", "attend", type="f16", heads=16, kv_heads=2, head_dim=64, page=16, seqs=5, new=1501, len=6007,
             spread=3, window=1000, sinks=16),
        # the last piece of a long prompt, grouped heads
        case("attend piece of a prompt", "attend", kv_heads=8, block=64, new=2048, len=8192),
        # a served batch behind one long instruction
        case("attend behind a prefix", "attend", kv_heads=8, page=128, block=64, seqs=64, len=17408, spread=8, prefix=16384),
        # a generated token of one sequence
        tables_case("tables of one sequence"),
        # a step of a served batch: most sequences get a token, some wait, some are over
        tables_case("tables of a batch's step", seqs=256, page=32, entries=512, held=16000, spread=16, idle=9, ended=17),
        # prompts of all lengths into a batch whose window gives pages back, more than there are pages for
        tables_case("tables of many prompts", seqs=1024, page=16, entries=1024, new=500, held=15000, spread=50, window=4096, sinks=4, ended=5, free=90),
    ]


def spread_int(rng, low, high):
    """Whole numbers whose logarithm is spread evenly; odd ones as often as even ones."""
    return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    while True:
        op = rng.choice(["append", "attend", "attend", "tables"])
        page = rng.choice([16, 32, 64, 128, 256])
        if op == "tables":
            seqs, entries = spread_int(rng, 1, 2048), spread_int(rng, 8, 4096)
            if seqs * entries > 1 << 20:
                continue
            prefix = rng.choice([0, 0, spread_int(rng, 1, 5000)])
            new = min(rng.choice([1, 1, spread_int(rng, 2, 8192)]), entries * page // 2, (1 << 19) // seqs)
            c = tables_case(None, seqs, page, entries, max(1, new), spread_int(rng, 1, entries * page // 2), rng.choice([0, 2, 16]), prefix=prefix,
                            idle=rng.choice([0, 0, 3, 9]), ended=rng.choice([0, 0, 4, 17]), free=rng.choice([50, 100, 150, 300]),
                            pad=rng.choice([1, 64, 256]))
            if rng.random() < 0.4:
                c.update(window=spread_int(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 16]))
            return c
        heads, kv_heads = rng.choice([(32, 32), (40, 40), (32, 8), (64, 8), (16, 2), (12, 4), (8, 1), (15, 5), (28, 4)])
        head_dim = rng.choice([64, 128, 128, 128, 256])
        type = rng.choice(["bf16", "f16"])
        block = rng.choice([b for b in (16, 32, 64, 128, 256) if b <= page])
        c = dict(type=type, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, block=block, spread=rng.choice([0, 2, 8]))
        if op == "append":
            new = rng.choice([1, spread_int(rng, 2, 8192)])
            c.update(x_type=rng.choice([type, type, "f32"]), seqs=spread_int(rng, 1, 256 if new == 1 else 8), new=new,
                     len=new + spread_int(rng, 30, 4096), rot=rng.choice([head_dim, head_dim, head_dim // 2]),
                     pairing=rng.choice(["halves", "neighbours"]))
        else:
            new = rng.choice([1, 1, spread_int(rng, 2, 16), spread_int(rng, 17, 4096)])
            c.update(seqs=spread_int(rng, 1, 128 if new == 1 else 8), new=new, len=new + spread_int(rng, 60, 131072 if new == 1 else 16384))
            if rng.random() < 0.4:
                c.update(window=spread_int(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 16]))
            if rng.random() < 0.3:
                c.update(seqs=spread_int(rng, 2, 128 if new == 1 else 8), prefix=spread_int(rng, 100, 32768))
                c["len"] += c["prefix"]
        c = case(None, op, **c)
        w = work(c)
        padded = c["seqs"] * c["new"] * c["heads"] * c["len"]
        if w["flops"] < 2.4e11 and w["bytes"] < 3e8 and c["seqs"] * c["len"] * c["kv_heads"] * c["head_dim"] < 1e9 and (op == "append" or padded < 6e8):
            return c


def lengths(c):
    """(new tokens, all tokens) of every sequence: the case's own, whatever the seed."""
    r = random.Random("%(seqs)d %(new)d %(len)d %(spread)d" % c)
    new, whole = [], []
    for b in range(c["seqs"]):
        ragged = c["spread"] and b  # the first sequence has the most of both
        n = r.randint(max(1, c["new"] // c["spread"]), c["new"]) if ragged else c["new"]
        own_part = c["len"] - c["prefix"]
        low = max(n, own_part // max(1, c["spread"]))
        new.append(n)
        whole.append(c["prefix"] + (n if c["new"] == own_part else r.randint(low, own_part) if ragged else own_part))
    return new, whole


def held_and_new(c):
    """(tokens held, tokens to come; -1: the sequence is over) of every sequence of a case of tables: the case's own."""
    r = random.Random("%(seqs)d %(new)d %(held)d %(spread)d" % c)
    held, new = [], []
    for b in range(c["seqs"]):
        ragged = c["spread"] and b
        held.append(c["prefix"] + (r.randint(c["held"] // c["spread"], c["held"]) if ragged else c["held"]))
        n = r.randint(max(1, c["new"] // c["spread"]), c["new"]) if ragged else c["new"]
        idle, ended = c["idle"] and b % c["idle"] == c["idle"] - 1, c["ended"] and b % c["ended"] == c["ended"] - 1
        new.append(-1 if ended else 0 if idle else n)
    return np.array(held), np.array(new)


def rows_of(c):
    n = int(held_and_new(c)[1].clip(min=0).sum())
    return max(1, -(-n // c["pad"]) * c["pad"])


def seen(c, first, last):
    """How many keys in [0, last] any of the rows at positions first .. last sees, and how many below the prefix's end."""
    low = max(0, first - c["window"] + 1) if c["window"] else 0
    sinks = min(c["sinks"], low)
    both = last + 1 - low + sinks
    shared = max(0, c["prefix"] - low) + min(sinks, c["prefix"])
    return both, shared


def work(c):
    if c["op"] == "tables":
        # the table read and written, held and new in, length and first row out, a place, a position and a sequence for each row, the pages that are taken
        entries, rows = c["seqs"] * c["entries"], rows_of(c)
        return {"bytes": 8 * entries + 16 * c["seqs"] + 16 * rows + 4 * (rows // c["page"]), "flops": 4 * entries + 4 * rows}
    new, whole = lengths(c)
    rows, d = sum(new), c["head_dim"]
    kv = 2 * c["kv_heads"] * (d + 4 / c["block"])  # bytes of a token
    if c["op"] == "append":
        x = TYPES[c["x_type"]].itemsize
        moved = rows * (c["heads"] * (x + 2) * d + 2 * c["kv_heads"] * x * d + kv)
        return {"bytes": int(moved) + len(set(p for n, w in zip(new, whole) for p in range(w - n, w))) * c["rot"] * 4 + c["seqs"] * 12,
                "flops": rows * (c["heads"] + c["kv_heads"]) * c["rot"] * 3}
    pairs = sum(sum(seen(c, p, p)[0] for p in range(w - n, w)) for n, w in zip(new, whole))
    reach = [seen(c, w - n, w - 1) for n, w in zip(new, whole)]
    private = sum(a - b for a, b in reach)
    prefix = max(b for a, b in reach)
    return {"bytes": int(rows * c["heads"] * (4 * d + 4) + (private + prefix) * kv) + c["seqs"] * 12, "flops": pairs * c["heads"] * d * 4}


def prepare(c, seed):
    return prepare_tables(c, seed) if c["op"] == "tables" else prepare_cache(c, seed)


def prepare_cache(c, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    t, d, page = TYPES[c["type"]], c["head_dim"], c["page"]
    new, whole = lengths(c)
    rows, prefix = sum(new), c["prefix"]
    private = [w - prefix for w in whole]
    stride = max(-(-p // page) for p in private)
    prefix_pages = -(-prefix // page)
    # pages in use: all for a cache without a window, else those with a token that a row can still see
    r = random.Random(seed)
    used = []
    for b, (n, w) in enumerate(zip(new, whole)):
        low = w - n - c["window"] + 1 if c["window"] and c["op"] != "append" else 0
        for i in range(-(-private[b] // page)):
            at = prefix + i * page
            if at + page > low or at < c["sinks"]:
                used.append((b, i))
    n_pages = prefix_pages + len(used) + 3
    order = list(range(n_pages))
    r.shuffle(order)
    table = torch.full((c["seqs"], stride), -1, dtype=torch.int32)
    if used:
        at = torch.tensor(used)
        table[at[:, 0], at[:, 1]] = torch.tensor(order[prefix_pages:prefix_pages + len(used)], dtype=torch.int32)
    shape = (n_pages, c["kv_heads"], page, d)
    # what earlier calls have left: numbers of about unit variance or half or twice that, block by block
    held = [(torch.randn(shape, device=dev, dtype=torch.bfloat16, generator=g) * 32).clamp_(-127, 127).to(torch.int8) for _ in range(2)]
    scales = [power_of_two(torch.randint(-6, -3, (n_pages, c["kv_heads"], page // c["block"]), device=dev, generator=g)) for _ in range(2)]
    st = {
        "case": c, "rows": rows, "k_cache": held[0], "v_cache": held[1], "k_scale": scales[0], "v_scale": scales[1],
        "pages": table.to(dev), "prefix_pages": torch.tensor(order[:prefix_pages], dtype=torch.int32, device=dev),
        "lens": torch.tensor(whole, dtype=torch.int32, device=dev),
        "starts": torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).to(dev),
    }
    if c["op"] == "append":
        x = TYPES[c["x_type"]]
        st["qkv"] = torch.randn((rows, c["heads"] + 2 * c["kv_heads"], d), device=dev, dtype=x, generator=g)
        # cosines and sines of every position, made once by the program
        half = c["rot"] // 2
        angle = torch.arange(c["len"], device=dev, dtype=torch.float64)[:, None] * torch.pow(
            10000.0, -torch.arange(half, device=dev, dtype=torch.float64) / half)
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        st["out"] = torch.empty((rows, c["heads"], d), device=dev, dtype=t)
    else:
        # a little more than unit variance: some rows look at few keys, most at many
        st["q"] = (torch.randn((rows, c["heads"], d), device=dev, dtype=torch.float32, generator=g) * 1.5).to(t)
        st["out"] = torch.empty((rows, c["heads"], d), device=dev, dtype=t)
        st["lse"] = torch.empty((rows, c["heads"]), device=dev, dtype=torch.float32)
    if own:  # the descriptions and the scratch memory that a program keeps beside its buffers
        import paper_2502_15443_amd as dc

        kind = {"bf16": dc.TYPE_BF16, "f16": dc.TYPE_F16, "f32": dc.TYPE_F32}
        st["dc"], st["stream"] = dc, torch.cuda.current_stream().cuda_stream
        st["cache"] = dc.KVCache(st["k_cache"], st["v_cache"], n_pages, c["kv_heads"], d, page, dc.TYPE_I8, rows_type=kind[c["type"]],
                                 scale_tokens=c["block"], k_scale_dev=st["k_scale"], v_scale_dev=st["v_scale"])
        st["batch"] = dc.KVBatch(c["seqs"], rows, c["new"], c["len"], st["lens"], st["pages"], stride,
                                 row_start_dev=None if c["new"] == 1 else st["starts"], prefix_len=prefix,
                                 prefix_pages_dev=st["prefix_pages"] if prefix else None)
        if c["op"] == "append":
            q, k, v = st["qkv"].split([c["heads"], c["kv_heads"], c["kv_heads"]], dim=1)
            st["new"] = dc.KVRows(kind[c["x_type"]], c["heads"], k, v, q, st["out"], rot_dim=c["rot"],
                                  pairing={"halves": dc.ROPE_HALVES, "neighbours": dc.ROPE_NEIGHBOURS}[c["pairing"]], cos_dev=st["cos"],
                                  sin_dev=st["sin"], n_positions=c["len"])
        else:
            st["attention"] = dc.Attention(c["heads"], st["q"], st["out"], st["lse"], d ** -0.5, window=c["window"], sinks=c["sinks"])
            n = dc.attention_paged_workspace(st["cache"], st["batch"], st["attention"])
            st["workspace"], st["workspace_bytes"] = torch.zeros(max(n, 16), dtype=torch.uint8, device=dev), n
    return st


def prepare_tables(c, seed):
    held, new = held_and_new(c)
    page, P, S = c["page"], c["prefix"], c["entries"]
    # the table that the step before has left: pages of the tokens held, but those behind the window of a row two pages back
    at = P + np.arange(S) * page
    there = at < held[:, None]
    if c["window"]:
        there &= (at + page > held[:, None] - 2 * page - c["window"]) | (at < c["sinks"])
    taken = int(sum(max(0, -(-(h + n - P) // page) - max(0, -(-(h - P) // page))) for h, n in zip(held, new) if n > 0))
    free = max(1, taken * c["free"] // 100)
    prefix_pages, used = -(-P // page), int(there.sum())
    n_pages = prefix_pages + used + free
    r = np.random.default_rng(seed)
    order = r.permutation(n_pages).astype(np.int32)
    table = np.full((c["seqs"], S), -1, dtype=np.int32)
    table[there] = order[prefix_pages:prefix_pages + used]
    first = int(r.integers(n_pages))
    ring = np.full(n_pages, -1, dtype=np.int32)
    ring[(first + np.arange(free)) % n_pages] = order[prefix_pages + used:]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rows = rows_of(c)
    st = {
        "case": c, "rows": rows, "n_pages": n_pages, "held": i32(held), "new": i32(new), "pages_in": i32(table), "prefix_pages": i32(order[:prefix_pages]),
        "free": i32(ring), "queue_in": i32([first, free]), "pages": torch.empty_like(i32(table)), "queue": i32([0, 0, 0]),
        "lens": i32(held), "starts": i32([0] * (c["seqs"] + 1)), "slots": torch.empty(rows, dtype=torch.int64, device="cuda"),
        "positions": i32([0] * rows), "row_seqs": i32([0] * rows),
    }
    if own:
        import paper_2502_15443_amd as dc

        st["dc"], st["stream"] = dc, torch.cuda.current_stream().cuda_stream
        st["requests"] = dc.KVRequests(c["seqs"], rows, page, S, n_pages, held_dev=st["held"], new_dev=st["new"], pages_in_dev=st["pages_in"],
                                       free_dev=st["free"], queue_in_dev=st["queue_in"], len_dev=st["lens"], row_start_dev=st["starts"],
                                       pages_dev=st["pages"], queue_dev=st["queue"], slot_dev=st["slots"], position_dev=st["positions"],
                                       seq_dev=st["row_seqs"], window=c["window"], sinks=c["sinks"], prefix_len=P,
                                       prefix_pages_dev=st["prefix_pages"] if P else None)
        n = dc.kv_tables_workspace(st["requests"])
        st["workspace"], st["workspace_bytes"] = torch.zeros(max(n, 16), dtype=torch.uint8, device="cuda"), n
    return st


def run(st):
    c = st["case"]
    if c["op"] == "tables":
        if own:
            st["dc"].kv_tables(st["requests"], st["workspace"], st["workspace_bytes"], st["stream"])
        else:
            plain_tables(st, c)
        return {name: st[name] for name in ("pages", "free", "queue", "lens", "starts", "slots", "positions", "row_seqs")}
    if c["op"] == "append":
        if own:
            st["dc"].kv_append(st["cache"], st["batch"], st["new"], st["stream"])
        else:
            plain_append(st, c)
        # whole numbers, and the scales that make them keys and values
        return {"q": st["out"], "k_cache": st["k_cache"], "v_cache": st["v_cache"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}
    if own:
        st["dc"].attention_paged(st["cache"], st["batch"], st["attention"], st["workspace"], st["workspace_bytes"], st["stream"])
        return {"out": st["out"], "lse": st["lse"]}
    out, lse = plain_attend(st, c)
    return {"out": out, "lse": lse}


# ---- the plain forms ----------------------------------------------------------------------------------------------------------

def places(st):
    """Sequence and position of every row."""
    row = torch.arange(st["rows"], device="cuda")
    seq = (row[:, None] >= st["starts"][None, 1:]).sum(1)
    return seq, st["lens"][seq] - st["starts"][seq + 1] + row


def turned(x, cos, sin, c):
    """x [rows, heads, d] in fp32 with its first rot values turned, pair by pair; every product and difference rounded."""
    rot = c["rot"]
    cos, sin = cos[:, None, :], sin[:, None, :]
    if c["pairing"] == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def power_of_two(e):
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def scale_of(most):
    """The smallest power of two, 2^-126 at least, of which 127 times is not below `most`."""
    part, exponent = torch.frexp(most)  # most = part 2^exponent, 127 = 127/128 2^7
    e = torch.where(part <= 127 / 128, exponent - 7, exponent - 6).clamp(min=-126)
    return power_of_two(torch.where(most > 0, e, -126))


def plain_append(st, c):
    seq, pos = places(st)
    q, k, v = st["qkv"].float().split([c["heads"], c["kv_heads"], c["kv_heads"]], dim=1)
    cos, sin = st["cos"][pos], st["sin"][pos]
    st["out"].copy_(turned(q, cos, sin, c))
    page, block, own_pos = c["page"], c["block"], pos - c["prefix"]
    at, place = st["pages"][seq, own_pos // page].long(), own_pos % page
    # the first row of each sequence: its block may hold earlier tokens, the others begin with a new one
    lead = st["starts"][:-1].long()
    l_at, l_block, l_place = at[lead], place[lead] // block, place[lead] % block
    old = l_block[:, None] * block + torch.arange(block, device="cuda")  # [seqs, block]
    earlier = torch.arange(block, device="cuda") < l_place[:, None]
    for x, held, scales in ((turned(k, cos, sin, c), st["k_cache"], st["k_scale"]), (v, st["v_cache"], st["v_scale"])):
        flat = scales.transpose(1, 2).reshape(-1, c["kv_heads"])  # a row to a block
        of_row = at * (page // block) + place // block
        before = flat[of_row[lead]]
        need = torch.zeros_like(flat).scatter_reduce_(0, of_row[:, None].expand(-1, c["kv_heads"]), x.abs().amax(-1), "amax")[of_row]
        scale = scale_of(need)
        joins = (of_row == of_row[lead][seq]) & (l_place > 0)[seq]  # the row's block holds earlier tokens
        scale = torch.where(joins[:, None], torch.maximum(scale, before[seq]), scale)
        now = scale[lead]
        values = held[l_at[:, None], :, old]  # [seqs, block, kv_heads, d]
        anew = torch.round(values.float() * (before * (1 / now))[:, None, :, None]).to(torch.int8)
        held[l_at[:, None], :, old] = torch.where(earlier[:, :, None, None], anew, values)
        held[at, :, place] = torch.round(x * (1 / scale)[..., None]).clamp(-127, 127).to(torch.int8)
        scales[at, :, place // block] = scale


def gathered(cache, scales, block, table):
    """[.., kv_heads, tokens, d] in fp32 of the pages of a table [.., pages]; absent pages give the values of page 0."""
    i = table.clamp(min=0).long()
    x = (cache[i].float() * scales[i].repeat_interleave(block, -1)[..., None]).transpose(-4, -3)
    return x.reshape(*x.shape[:-3], -1, x.shape[-1])


def plain_attend(st, c):
    B, H, KV, d, page, P = c["seqs"], c["heads"], c["kv_heads"], c["head_dim"], c["page"], c["prefix"]
    Q, block = c["new"], c["block"]
    keys, values = (st["k_cache"], st["k_scale"], block), (st["v_cache"], st["v_scale"], block)
    i = torch.arange(Q, device="cuda")
    count = (st["starts"][1:] - st["starts"][:-1])[:, None]
    row = (st["starts"][:-1, None] + i).clamp(max=st["rows"] - 1)  # [B, Q]: the rows of every sequence, and others where it has fewer
    pos = st["lens"][:, None] - count + i
    q = st["q"].float()[row].reshape(B, Q, KV, H // KV, d).permute(0, 2, 3, 1, 4).reshape(B, KV, -1, d) * d ** -0.5  # [B, KV, G*Q, d]

    def visible(key, there):  # key positions [T], there [B or 1, T] -> [B, Q, T]
        key, p = key[None, None, :], pos[:, :, None]
        ok = (key <= p) & there[:, None, :]
        return ok & ((key > p - c["window"]) | (key < c["sinks"])) if c["window"] else ok

    T = st["pages"].shape[1] * page
    key = P + torch.arange(T, device="cuda")
    mask = visible(key, (st["pages"] >= 0).repeat_interleave(page, 1))
    s = q @ gathered(*keys, st["pages"]).transpose(-1, -2).contiguous()  # [B, KV, G*Q, T]
    s = s.reshape(B, KV, H // KV, Q, T).masked_fill_(~mask[:, None, None], -math.inf).reshape(B, KV, -1, T)
    top = s.amax(-1, keepdim=True)
    if P:
        mask = visible(torch.arange(P, device="cuda"), torch.ones((1, P), dtype=torch.bool, device="cuda"))
        k, v = gathered(*keys, st["prefix_pages"])[:, :P], gathered(*values, st["prefix_pages"])[:, :P]
        sp = q.transpose(0, 1).reshape(KV, -1, d) @ k.transpose(-1, -2).contiguous()  # [KV, B*G*Q, P]
        sp = sp.reshape(KV, B, H // KV, Q, P).masked_fill_(~mask[None, :, None], -math.inf).reshape(KV, B, -1, P)
        top = torch.maximum(top, sp.amax(-1, keepdim=True).transpose(0, 1))
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = s.sub_(top).exp_()
    total, out = e.sum(-1, keepdim=True), e @ gathered(*values, st["pages"])
    if P:
        ep = sp.sub_(top.transpose(0, 1)).exp_()
        total += ep.sum(-1, keepdim=True).transpose(0, 1)
        out += (ep.reshape(KV, -1, P) @ v).reshape(KV, B, -1, d).transpose(0, 1)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    lse = top + total.log()
    own_rows = i < count
    out = out.reshape(B, KV, H // KV, Q, d).permute(0, 3, 1, 2, 4).reshape(B, Q, H, d)[own_rows]
    lse = lse.reshape(B, KV, H // KV, Q).permute(0, 3, 1, 2).reshape(B, Q, H)[own_rows]
    return out.to(TYPES[c["type"]]), lse


def plain_tables(st, c):
    page, P, S, n_pages = c["page"], c["prefix"], c["entries"], st["n_pages"]
    over = st["new"] < 0
    held = torch.where(over, 0, st["held"].clamp(min=0)).long()
    starts = torch.cat([st["starts"][:1] * 0, st["new"].clamp(min=0).cumsum(0)]).clamp(max=st["rows"])
    lens = held + starts[1:] - starts[:-1]
    at = P + torch.arange(S, device="cuda") * page  # first position of each entry
    wanted = at < (held + st["new"].clamp(min=0))[:, None]
    if c["window"]:
        wanted &= (at + page - 1 > held[:, None] - c["window"]) | (at < c["sinks"])
    before = st["pages_in"]
    there = (before >= 0) & (before < n_pages)
    first, count = st["queue_in"][0].long(), st["queue_in"][1].long()
    take = wanted & ~there & (at >= held[:, None])
    rank = take.flatten().cumsum(0).reshape(take.shape) - 1
    got = take & (rank < count)
    pages = torch.where(wanted & there, before, torch.where(got, st["free"][(first + rank.clamp(min=0)) % n_pages], -1))
    back = there & ~wanted
    rank_back = back.flatten().cumsum(0).reshape(back.shape) - 1
    # every place behind the free ones gets the page with that number among those that go back; the others keep what they hold
    nth = torch.full((n_pages + 1,), -1, dtype=torch.int32, device="cuda").scatter_(0, torch.where(back, rank_back, n_pages).flatten(), before.flatten())
    behind = (torch.arange(n_pages, device="cuda") - first - count) % n_pages
    st["free"].copy_(torch.where(behind < back.sum(), nth[behind], st["free"]))
    st["queue"].copy_(torch.stack([(first + got.sum()) % n_pages, count - got.sum() + back.sum(), take.sum() - got.sum()]))
    st["pages"].copy_(pages)
    st["lens"].copy_(lens)
    st["starts"].copy_(starts)
    row = torch.arange(st["rows"], device="cuda")
    seq = (row[:, None] >= starts[None, 1:]).sum(1)
    is_row = seq < c["seqs"]
    s = seq.clamp(max=c["seqs"] - 1)
    pos = held[s] + row - starts[s]
    entry = (pos - P) // page
    of = torch.where(entry < S, pages[s, entry.clamp(0, S - 1)], -1)
    place = pos - P - entry * page
    if P:
        in_prefix = pos < P
        of = torch.where(in_prefix, st["prefix_pages"][(pos // page).clamp(max=len(st["prefix_pages"]) - 1)], of)
        place = torch.where(in_prefix, pos % page, place)
    st["slots"].copy_(torch.where(is_row & (of >= 0), of.long() * page + place, -1))
    st["positions"].copy_(torch.where(is_row, pos, -1))
    st["row_seqs"].copy_(torch.where(is_row, seq, -1))


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------------

def exact(c, seed):
    if c["op"] == "tables":
        return None  # whole numbers
    st = prepare(c, seed)
    new, whole = lengths(c)
    page, block, KV, G = c["page"], c["block"], c["kv_heads"], c["heads"] // c["kv_heads"]
    table, prefix_table = st["pages"].cpu(), st["prefix_pages"].cpu()
    first = 0
    if c["op"] == "append":
        scales = {"k": st["k_scale"].double(), "v": st["v_scale"].double()}
        q_out = torch.empty(st["out"].shape, dtype=torch.float64, device="cuda")
        half = c["rot"] // 2
        for b, (n, w) in enumerate(zip(new, whole)):
            x = st["qkv"][first:first + n].double()
            # the pair (a, b) as a complex number times cos + i sin
            turn = torch.complex(st["cos"][w - n:w].double(), st["sin"][w - n:w].double())[:, None]
            pairs = x[:, :, :c["rot"]]
            pairs = pairs.reshape(n, -1, 2, half).transpose(2, 3) if c["pairing"] == "halves" else pairs.reshape(n, -1, half, 2)
            pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            pairs = pairs.transpose(2, 3) if c["pairing"] == "halves" else pairs
            qk = torch.cat([pairs.reshape(n, -1, c["rot"]), x[:, :, c["rot"]:]], -1)
            q_out[first:first + n] = qk[:, :c["heads"]]
            parts = {"k": qk[:, c["heads"]:c["heads"] + KV].abs().amax(-1), "v": x[:, c["heads"] + KV:].abs().amax(-1)}
            # the sequence's blocks from the first new token's on, each as many rows as it has new tokens
            places = torch.arange(w - n - c["prefix"], w - c["prefix"])
            number = (places // block - places[0] // block).cuda()
            count = int(number[-1]) + 1
            inside = torch.arange(count) + places[0] // block
            at, i = table[b][inside * block // page].long().cuda(), (inside % (page // block)).cuda()
            for name, most in parts.items():
                need = torch.zeros((count, KV), dtype=torch.float64, device="cuda").index_reduce_(0, number, most, "amax")
                s = torch.exp2(torch.ceil(torch.log2(need / 127)).clamp(min=-126))
                if places[0] % block:
                    s[0] = torch.maximum(s[0], scales[name][at[0], :, i[0]])
                scales[name][at, :, i] = s
            first += n
        return {"q": q_out, "k_cache": None, "v_cache": None, "k_scale": scales["k"], "v_scale": scales["v"]}
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    for b, (n, w) in enumerate(zip(new, whole)):
        # page and place of every position that is held
        at = torch.full((w,), -1, dtype=torch.long)
        pos = torch.arange(w)
        at[:c["prefix"]] = prefix_table[pos[:c["prefix"]] // page].long()
        at[c["prefix"]:] = table[b][(pos[c["prefix"]:] - c["prefix"]) // page].long()
        place = torch.where(pos < c["prefix"], pos % page, (pos - c["prefix"]) % page)
        held = (at >= 0).nonzero().flatten()
        at, place, key = at[held].cuda(), place[held].cuda(), held.cuda()
        p = torch.arange(w - n, w, device="cuda")[:, None]
        hidden = key[None, :] > p
        if c["window"]:
            hidden |= (key[None, :] <= p - c["window"]) & (key[None, :] >= c["sinks"])
        for h in range(KV):
            k = st["k_cache"][at, h, place].double() * st["k_scale"][at, h, place // block].double()[:, None]
            v = st["v_cache"][at, h, place].double() * st["v_scale"][at, h, place // block].double()[:, None]
            q = st["q"][first:first + n, h * G:(h + 1) * G].double()
            for j in range(G):
                s = (q[:, j] @ k.t()) / math.sqrt(c["head_dim"])
                s[hidden] = -math.inf
                l = torch.logsumexp(s, 1)
                out[first:first + n, h * G + j] = torch.exp(s - l[:, None]) @ v
                lse[first:first + n, h * G + j] = l
        first += n
    return {"out": out, "lse": lse}
