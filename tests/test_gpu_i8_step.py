"""Tables of pages, append to a cache of 8 bits and attention over it, as a program runs them: step after step, from arrays that stay on the GPU, eagerly and as a
recorded graph whose rows are padded.  Sequences begin, grow, wait and end; every step is compared with the oracles."""
import importlib.util
import os

import numpy as np
import pytest

import oracle.attention as oa
import oracle.cache_i8 as oc8
import oracle.tables as ot
import paper_2502_15443_amd as dc
from tests.attention_cases import f64
from tests.i8_cases import check_attend_i8
from tests.test_gpu_kv_append import angles

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("recorded", [False, True])
@pytest.mark.parametrize("window,sinks,prefix", [(0, 0, 0), (40, 4, 0), (0, 0, 21), (50, 30, 21)])
def test_steps_of_a_served_batch(recorded, window, sinks, prefix):
    print(f"case steps recorded={recorded} window={window} prefix={prefix}", flush=True)
    r = np.random.default_rng(1)
    seqs, heads, kv, d, page, block, entries, n_pages, rows, max_new, steps = 5, 4, 2, 64, 16, 16, 10, 60, 64, 30, 14
    prefix_pages = np.array([7, 50][:-(-prefix // page)], dtype=np.int32)
    cos, sin = angles(200, d // 2)
    cd, sd = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    pools = [r.integers(-127, 128, (n_pages, kv, page, d)).astype(np.int8) for _ in range(2)]
    scales = [(2.0 ** r.integers(-6, -3, (n_pages, kv, 1))).astype(np.float32) for _ in range(2)]  # the prefix's are sound, the others are never read
    for s in scales:
        s[[p for p in range(n_pages) if p not in prefix_pages]] = np.nan
    free = [int(p) for p in r.permutation(n_pages) if p not in prefix_pages]
    state = {"held": [prefix] * seqs, "pages": [[-1] * entries for _ in range(seqs)], "free": free + [-1] * (n_pages - len(free)), "queue": (0, len(free))}

    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(np.array(a, dtype=np.int32))).cuda()  # noqa: E731
    t = {n: i32(v) for n, v in (("lens", state["held"]), ("new", [0] * seqs), ("pages", state["pages"]), ("free", state["free"]),
                                ("queue", [*state["queue"], 0]), ("starts", [0] * (seqs + 1)), ("positions", [0] * rows), ("seqs", [0] * rows))}
    t["slots"], t["prefix"] = torch.zeros(rows, dtype=torch.int64, device="cuda"), i32(prefix_pages)
    held = [torch.from_numpy(a.copy()).cuda() for a in pools + scales]
    x = torch.zeros((rows, heads + 2 * kv, d), device="cuda")
    turned, out = (torch.zeros((rows, heads, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.zeros((rows, heads), device="cuda")
    q = dc.KVRequests(seqs, rows, page, entries, n_pages, held_dev=t["lens"], new_dev=t["new"], pages_in_dev=t["pages"], queue_in_dev=t["queue"], free_dev=t["free"],
                      len_dev=t["lens"], row_start_dev=t["starts"], pages_dev=t["pages"], queue_dev=t["queue"], slot_dev=t["slots"], position_dev=t["positions"],
                      seq_dev=t["seqs"], window=window, sinks=sinks, prefix_len=prefix, prefix_pages_dev=t["prefix"] if prefix else None)
    cache = dc.KVCache(held[0], held[1], n_pages, kv, d, page, dc.TYPE_I8, scale_tokens=block, k_scale_dev=held[2], v_scale_dev=held[3])
    batch = dc.KVBatch(seqs, rows, max_new, 150, t["lens"], t["pages"], entries, row_start_dev=t["starts"], prefix_len=prefix,
                       prefix_pages_dev=t["prefix"] if prefix else None)
    new_rows = dc.KVRows(dc.TYPE_F32, heads, x[:, heads:heads + kv], x[:, heads + kv:], x[:, :heads], turned, rot_dim=d, cos_dev=cd, sin_dev=sd, n_positions=200,
                         position_dev=t["positions"])
    attention = dc.Attention(heads, turned, out, lse, d ** -0.5, window=window, sinks=sinks)
    n_tables, n_attention = dc.kv_tables_workspace(q), dc.attention_paged_workspace(cache, batch, attention)
    ws_tables, ws_attention = (torch.empty(n + 16, dtype=torch.uint8, device="cuda") for n in (n_tables, n_attention))

    def step(stream):
        dc.kv_tables(q, ws_tables, n_tables, stream)
        dc.kv_append(cache, batch, new_rows, stream)
        dc.attention_paged(cache, batch, attention, ws_attention, n_attention, stream)

    graph = None
    if recorded:
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step(side.cuda_stream)
    for number in range(steps):
        h = state["held"]
        new = [-1 if n > prefix + 90 else int(r.choice([0, 1, 1, 1, r.integers(2, max_new + 1)])) for n in h]
        while sum(max(n, 0) for n in new) > rows:
            new[new.index(max(new))] = 1
        rows_now = r.standard_normal((rows, heads + 2 * kv, d)).astype(np.float32) * np.float32(2.0) ** r.integers(-2, 3, (rows, 1, 1))
        x.copy_(torch.from_numpy(rows_now.astype(np.float32)))
        t["new"].copy_(i32(new))
        for b, n in enumerate(new):  # a sequence that is over gives way to one that begins
            if h[b] == 0:
                t["lens"][b] = prefix
                h[b] = prefix
        out.fill_(7.75), lse.fill_(7.75)
        torch.cuda.synchronize()
        if graph:
            graph.replay()
        else:
            step(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        want = ot.tables(h, new, state["pages"], state["free"], state["queue"], rows, page, n_pages, prefix, prefix_pages, window, sinks)
        for name, key in (("pages", "pages"), ("free", "free"), ("queue", "queue"), ("lens", "lens"), ("starts", "starts"), ("slots", "slots"),
                          ("positions", "positions"), ("seqs", "seqs")):
            assert t[name].flatten().tolist() == np.array(want[key]).flatten().tolist(), (number, name)
        state = {"held": list(want["lens"]), "pages": want["pages"], "free": want["free"], "queue": tuple(want["queue"][:2])}
        now = {"lens": want["lens"], "starts": want["starts"], "pages": np.array(want["pages"]), "prefix_len": prefix, "prefix_pages": prefix_pages}
        # rows without a sequence have position -1 and are left alone
        pools_and_scales = oc8.append(*pools, *scales, now, block, rows_now[:, heads:heads + kv], rows_now[:, heads + kv:], cos, sin, False)
        pools, scales = list(pools_and_scales[:2]), list(pools_and_scales[2:])
        for got, w in zip(held, pools + scales):
            assert np.array_equal(got.cpu().numpy().view(np.uint8), w.view(np.uint8)), number
        ref, ref_lse, size = oa.attend(oc8.values(pools[0], scales[0]), oc8.values(pools[1], scales[1]), now, f64(turned), np.float64(np.float32(d ** -0.5)), window, sinks)
        total = want["starts"][-1]
        check_attend_i8("bf16", d, f64(out)[:total], f64(lse)[:total], ref[:total], ref_lse[:total], {n: s[:total] for n, s in size.items()}, 2.0)
        assert (out[total:] == 7.75).all() and (lse[total:] == 7.75).all()


def test_two_recorded_steps_share_their_workspace():
    """Two graphs, of generated tokens and of a prompt, over one cache and one workspace, replayed by turns."""
    from tests.attention_cases import device_batch
    from tests.i8_cases import device_cache_i8, paged_i8, pool_values

    p = paged_i8(3, 2, 128, 64, 32, [900, 300], [1, 1])
    prompt = dict(p, news=[150, 70], batch=dict(p["batch"], starts=np.array([0, 150, 220], dtype=np.int32)))
    cache, t = device_cache_i8(p)
    problems, most = [], 0
    for one in (p, prompt):
        rows = int(one["batch"]["starts"][-1])
        q = torch.from_numpy(p["rng"].standard_normal((rows, 8, 128)).astype(np.float32)).to(torch.bfloat16).cuda()
        out, lse = torch.empty_like(q), torch.empty((rows, 8), device="cuda")
        b, a = device_batch(one), dc.Attention(8, q, out, lse, 0.1)
        n = dc.attention_paged_workspace(cache, b, a)
        most = max(most, n)
        problems.append((one, q, out, lse, b, a, n))
    ws = torch.empty(most + 16, dtype=torch.uint8, device="cuda")
    graphs, side = [], torch.cuda.Stream()
    torch.cuda.synchronize()
    for *_, b, a, n in problems:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            dc.attention_paged(cache, b, a, ws, n, side.cuda_stream)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for one, q, out, lse, *_ in problems:
        ref, ref_lse, size = oa.attend(*pool_values(p), one["batch"], f64(q), np.float64(np.float32(0.1)))
        check_attend_i8("bf16", 128, f64(out), f64(lse), ref, ref_lse, size, 2.0 ** -4)


def test_the_example_holds_what_it_holds_in_16_bits():
    """The decoder layer with a cache of 8 bits: a prompt, then tokens.  Keys and values of the prompt are those of the bf16 cache, up to a rounding to
    bf16 there (2^-8) and here to half a step; what the tokens' output is made of runs through them."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_layer.py")
    spec = importlib.util.spec_from_file_location("decoder_layer_example_i8", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    n, hidden, table = 130, 512, [[5, 0, 3]]
    x = torch.randn(n, hidden, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    layers = [example.DecoderLayer(hidden, 8, 2, 1024, 8, n, seed=3, cache=c) for c in ("bf16", "i8")]
    results = [layer.prompt(x[:100], example.batch_of([100], [100], table)) for layer in layers]
    torch.cuda.synchronize()
    plain, eight = layers
    for pool, wide, scale in ((eight.k_pool, plain.k_pool, eight.k_scale), (eight.v_pool, plain.v_pool, eight.v_scale)):
        for page in table[0][:2]:
            tokens = 64 if page == 5 else 36
            s = scale[page].repeat_interleave(example.SCALE_TOKENS, 1)[:, :tokens, None]
            off = (pool[page, :, :tokens].float() * s - wide[page, :, :tokens].float()).abs()
            assert (off <= 0.5 * s + 2.0 ** -8 * wide[page, :, :tokens].float().abs()).all()
    tokens = [layer.token(x[t:t + 1], example.batch_of([t + 1], [1], table)) for t in range(100, n) for layer in layers]
    assert all(torch.isfinite(y).all() for y in results + tokens)
