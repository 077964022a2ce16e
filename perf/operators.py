"""Operator cases: what a decoder layer does between its products, over a cache of keys and values in pages.

A program that keeps its INT8 weights compressed multiplies them with `dc.decompress_gemv_layer` (or from the decompression
buffer).  Between the query/key/value products and the output product a layer turns queries and keys by their position, puts
keys and values into its cache, and attends over the cache.  Three kinds of case:

* ``append``: rotary positions on queries and keys, keys and values into the pages of their sequences.  The rows are slices of one
  fused query/key/value row, as the products leave them, in fp32 (the products' accumulators) or in 16 bits.
* ``attend``: causal attention of the new tokens over the cache, with or without a sliding window whose first tokens (sinks) stay
  visible: one token a sequence (a step of generation), whole prompts, and pieces of prompts.  Pages that no row can see any more
  have been given back: their table entries are -1.
* ``shared``: the same for a batch whose sequences begin with the same long prefix, held once.

Heads, head sizes and layer shapes are those of Llama-7B and Llama-13B (32 and 40 heads of 128) and generic grouped ones.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def case(name, op, type="bf16", x_type="bf16", heads=32, kv_heads=32, head_dim=128, page=64, seqs=1, new=1, len=1024, spread=0,
         window=0, sinks=0, prefix=0, rot=0, pairing="halves"):
    c = dict(op=op, type=type, x_type=x_type, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, seqs=seqs, new=new,
             len=len, spread=spread, window=window, sinks=sinks, prefix=prefix, rot=rot, pairing=pairing)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a generated token of Llama-7B, straight from the products' fp32 results: latency is all
        case("append one token", "append", x_type="f32", len=1000, rot=128),
        # a step of a served batch with grouped heads
        case("append batch of tokens", "append", kv_heads=8, seqs=96, len=4000, spread=8, rot=128),
        # the prompt of Llama-13B
        case("append long prompt", "append", heads=40, kv_heads=40, page=128, new=8192, len=8192, rot=128),
        # prompts of odd lengths behind tokens that are already there; half of the head is turned, neighbours in pairs
        case("append ragged pieces", "append", type="f16", x_type="f16", heads=16, kv_heads=2, head_dim=64, page=16, seqs=7, new=777,
             len=2001, spread=4, rot=32, pairing="neighbours"),
        # a generated token of Llama-7B
        case("attend one token", "attend", len=1999),
        # one token over a very long context
        case("attend token, long context", "attend", heads=64, kv_heads=8, page=128, len=131071),
        # a step of a served batch, contexts of all lengths
        case("attend batch of tokens", "attend", kv_heads=8, page=32, seqs=64, len=8192, spread=16),
        # streaming generation of Llama-13B: window and sinks, the pages between given back
        case("attend window and sinks", "attend", type="f16", heads=40, kv_heads=40, page=16, seqs=8, len=30011, spread=2, window=4096,
             sinks=4),
        # the prompt of Llama-7B
        case("attend long prompt", "attend", new=8192, len=8192),
        # pieces of prompts through a window, small heads, odd lengths
        case("attend ragged pieces", "attend", type="f16", heads=16, kv_heads=2, head_dim=64, page=16, seqs=5, new=1501, len=6007,
             spread=3, window=1000, sinks=16),
        # several answers to one question, Llama-7B
        case("shared short prefix", "shared", seqs=8, len=700, spread=4, prefix=500),
        # a served batch behind one long instruction
        case("shared long prefix", "shared", kv_heads=8, page=128, seqs=64, len=17408, spread=8, prefix=16384),
    ]


def spread_int(rng, low, high):
    """Whole numbers whose logarithm is spread evenly; odd ones as often as even ones."""
    return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    while True:
        op = rng.choice(["append", "attend", "attend", "shared"])
        heads, kv_heads = rng.choice([(32, 32), (40, 40), (32, 8), (64, 8), (16, 2), (12, 4), (8, 1), (15, 5), (28, 4)])
        head_dim = rng.choice([64, 128, 128, 128, 256])
        type = rng.choice(["bf16", "f16"])
        page = rng.choice([16, 32, 64, 128, 256])
        c = dict(type=type, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, spread=rng.choice([0, 2, 8]))
        if op == "append":
            new = rng.choice([1, spread_int(rng, 2, 8192)])
            c.update(x_type=rng.choice([type, type, "f32"]), seqs=spread_int(rng, 1, 256 if new == 1 else 8), new=new,
                     len=new + spread_int(rng, 30, 4096), rot=rng.choice([head_dim, head_dim, head_dim // 2]),
                     pairing=rng.choice(["halves", "neighbours"]))
        else:
            new = rng.choice([1, 1, spread_int(rng, 2, 16), spread_int(rng, 17, 8192)])
            c.update(seqs=spread_int(rng, 1, 128 if new == 1 else 8), new=new, len=new + spread_int(rng, 60, 131072 if new == 1 else 16384))
            if rng.random() < 0.4:
                c.update(window=spread_int(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 16]))
            if op == "shared":
                c.update(seqs=spread_int(rng, 2, 128 if new == 1 else 8), prefix=spread_int(rng, 100, 32768))
                c["len"] += c["prefix"]
        c = case(None, op, **c)
        w = work(c)
        padded = c["seqs"] * c["new"] * c["heads"] * c["len"]
        if w["flops"] < 5e11 and w["bytes"] < 5e8 and c["seqs"] * c["len"] * c["kv_heads"] * c["head_dim"] < 2e9 and (op == "append" or padded < 2.1e9):
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


def seen(c, first, last):
    """How many keys in [0, last] any of the rows at positions first .. last sees, and how many below the prefix's end."""
    low = max(0, first - c["window"] + 1) if c["window"] else 0
    sinks = min(c["sinks"], low)
    both = last + 1 - low + sinks
    shared = max(0, c["prefix"] - low) + min(sinks, c["prefix"])
    return both, shared


def work(c):
    new, whole = lengths(c)
    rows, d, size = sum(new), c["head_dim"], 2
    if c["op"] == "append":
        x = TYPES[c["x_type"]].itemsize
        moved = rows * (c["heads"] + 2 * c["kv_heads"]) * d
        return {"bytes": moved * (x + size) + len(set(p for n, w in zip(new, whole) for p in range(w - n, w))) * c["rot"] * 4
                + c["seqs"] * 12, "flops": rows * (c["heads"] + c["kv_heads"]) * c["rot"] * 3}
    kv = 2 * c["kv_heads"] * d * size
    pairs = sum(sum(seen(c, p, p)[0] for p in range(w - n, w)) for n, w in zip(new, whole))
    reach = [seen(c, w - n, w - 1) for n, w in zip(new, whole)]
    private = sum(a - b for a, b in reach)
    prefix = max(b for a, b in reach)
    return {"bytes": rows * c["heads"] * (2 * d * size + 4) + (private + prefix) * kv + c["seqs"] * 12, "flops": pairs * c["heads"] * d * 4}


def prepare(c, seed):
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
    st = {
        "case": c, "rows": rows,
        "k_cache": torch.randn(shape, device=dev, dtype=t, generator=g), "v_cache": torch.randn(shape, device=dev, dtype=t, generator=g),
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
        st["cache"] = dc.KVCache(st["k_cache"], st["v_cache"], n_pages, c["kv_heads"], d, page, kind[c["type"]])
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


def run(st):
    c = st["case"]
    if c["op"] == "append":
        if own:
            st["dc"].kv_append(st["cache"], st["batch"], st["new"], st["stream"])
        else:
            plain_append(st, c)
        return {"q": st["out"], "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
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
    """x [rows, heads, d] in fp32 with its first rot values turned, pair by pair."""
    rot = c["rot"]
    cos, sin = cos[:, None, :], sin[:, None, :]
    if c["pairing"] == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def plain_append(st, c):
    seq, pos = places(st)
    q, k, v = st["qkv"].float().split([c["heads"], c["kv_heads"], c["kv_heads"]], dim=1)
    cos, sin = st["cos"][pos], st["sin"][pos]
    st["out"].copy_(turned(q, cos, sin, c))
    at, t = st["pages"][seq, (pos - c["prefix"]) // c["page"]].long(), (pos - c["prefix"]) % c["page"]
    st["k_cache"][at, :, t] = turned(k, cos, sin, c).to(st["k_cache"].dtype)
    st["v_cache"][at, :, t] = v.to(st["v_cache"].dtype)


def gathered(cache, table):
    """[.., kv_heads, tokens, d] in fp32 of the pages of a table [.., pages]; absent pages give the values of page 0."""
    x = cache[table.clamp(min=0).long()].float().transpose(-4, -3)
    return x.reshape(*x.shape[:-3], -1, x.shape[-1])


def plain_attend(st, c):
    B, H, KV, d, page, P = c["seqs"], c["heads"], c["kv_heads"], c["head_dim"], c["page"], c["prefix"]
    Q = c["new"]
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
    s = q @ gathered(st["k_cache"], st["pages"]).transpose(-1, -2).contiguous()  # [B, KV, G*Q, T]
    s = s.reshape(B, KV, H // KV, Q, T).masked_fill_(~mask[:, None, None], -math.inf).reshape(B, KV, -1, T)
    top = s.amax(-1, keepdim=True)
    if P:
        mask = visible(torch.arange(P, device="cuda"), torch.ones((1, P), dtype=torch.bool, device="cuda"))
        k, v = gathered(st["k_cache"], st["prefix_pages"])[:, :P], gathered(st["v_cache"], st["prefix_pages"])[:, :P]
        sp = q.transpose(0, 1).reshape(KV, -1, d) @ k.transpose(-1, -2).contiguous()  # [KV, B*G*Q, P]
        sp = sp.reshape(KV, B, H // KV, Q, P).masked_fill_(~mask[None, :, None], -math.inf).reshape(KV, B, -1, P)
        top = torch.maximum(top, sp.amax(-1, keepdim=True).transpose(0, 1))
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = s.sub_(top).exp_()
    total, out = e.sum(-1, keepdim=True), e @ gathered(st["v_cache"], st["pages"])
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


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------------

def exact(c, seed):
    st = prepare(c, seed)
    new, whole = lengths(c)
    page, KV, G = c["page"], c["kv_heads"], c["heads"] // c["kv_heads"]
    K, V = st["k_cache"], st["v_cache"]
    table, prefix_table = st["pages"].cpu(), st["prefix_pages"].cpu()
    first = 0
    if c["op"] == "append":
        K, V = K.double(), V.double()
        q_out = torch.empty(st["out"].shape, dtype=torch.float64, device="cuda")
        half = c["rot"] // 2
        for b, (n, w) in enumerate(zip(new, whole)):
            pos = torch.arange(w - n, w)
            x = st["qkv"][first:first + n].double()
            # the pair (a, b) as a complex number times cos + i sin
            turn = torch.complex(st["cos"][w - n:w].double(), st["sin"][w - n:w].double())[:, None]
            pairs = x[:, :, :c["rot"]]
            pairs = pairs.reshape(n, -1, 2, half).transpose(2, 3) if c["pairing"] == "halves" else pairs.reshape(n, -1, half, 2)
            pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            pairs = pairs.transpose(2, 3) if c["pairing"] == "halves" else pairs
            qk = torch.cat([pairs.reshape(n, -1, c["rot"]), x[:, :, c["rot"]:]], -1)
            q_out[first:first + n] = qk[:, :c["heads"]]
            at, t = table[b][(pos - c["prefix"]) // page].long().cuda(), ((pos - c["prefix"]) % page).cuda()
            K[at, :, t] = qk[:, c["heads"]:c["heads"] + KV]
            V[at, :, t] = x[:, c["heads"] + KV:]
            first += n
        return {"q": q_out, "k_cache": K, "v_cache": V}
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
            k, v = K[at, h, place].double(), V[at, h, place].double()
            q = st["q"][first:first + n, h * G:(h + 1) * G].double()
            for j in range(G):
                s = (q[:, j] @ k.t()) / math.sqrt(c["head_dim"])
                s[hidden] = -math.inf
                l = torch.logsumexp(s, 1)
                out[first:first + n, h * G + j] = torch.exp(s - l[:, None]) @ v
                lse[first:first + n, h * G + j] = l
        first += n
    return {"out": out, "lse": lse}
