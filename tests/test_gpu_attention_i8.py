"""dc_attention_paged over a cache of 8 bits against the oracle in 64 bits through the C ABI: types, head sizes and groups, blocks and pages, lengths from
nothing to several tiles, windows and sinks, absent pages, common prefixes, layouts, and what must have no influence (numbers of no token are any bytes,
scales of blocks without tokens are no sound ones)."""
import numpy as np
import pytest

import oracle.attention as oa
import paper_2502_15443_amd as dc
from tests.attention_cases import device_batch, f64, rows_tensor, torch_type
from tests.i8_cases import check_attend_i8, device_cache_i8, paged_i8, pool_values

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SENTINEL = 7.75


def attend(p, heads, q, scale, window=0, sinks=0, layout="dense", uniform=False, max_len=None, stream=None):
    """(out, lse) as fp64 arrays; checks that nothing outside the rows was written."""
    cache, t = device_cache_i8(p)
    batch = device_batch(p, uniform, max_len)
    rows, d = q.shape[0], p["head_dim"]
    qd = rows_tensor(q.cuda(), layout)
    wide = torch.full((rows + 2, heads + 2, d), SENTINEL, dtype=q.dtype, device="cuda")
    out = wide[1:-1, 1:-1]
    lse = torch.full((rows + 2, heads), SENTINEL, dtype=torch.float32, device="cuda")
    a = dc.Attention(heads, qd, out, lse[1:-1], scale, window=window, sinks=sinks)
    n = dc.attention_paged_workspace(cache, batch, a)
    ws = torch.full((max(n, 16) + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    dc.attention_paged(cache, batch, a, ws if n else None, n, torch.cuda.current_stream().cuda_stream if stream is None else stream.cuda_stream)
    torch.cuda.synchronize()
    assert (ws[n:] == 0xFF).all()
    edge = wide.clone()
    edge[1:-1, 1:-1] = SENTINEL
    assert (edge == SENTINEL).all() and (lse[0] == SENTINEL).all() and (lse[-1] == SENTINEL).all()
    assert all(np.array_equal(a.cpu().numpy().view(np.uint8), p[n].view(np.uint8)) for a, n in zip(t, ("k", "v", "ks", "vs")))
    return f64(out), f64(lse[1:-1])


def queries(p, heads):
    rows = int(p["batch"]["starts"][-1])
    return torch.from_numpy(p["rng"].standard_normal((rows, heads, p["head_dim"])).astype(np.float32) * 1.5).to(torch_type(p["type"]))


def run(seed, type, heads, kv_heads, d, page, block, lens, news, window=0, sinks=0, prefix=0, absent=(), scale=None, scales=(-6, -4), q=None, **how):
    print(f"case attention i8 {type} heads={heads}/{kv_heads} d={d} page={page} block={block} lens={lens} news={news} window={window} sinks={sinks} "
          f"prefix={prefix} absent={absent} {how}", flush=True)
    p = paged_i8(seed, kv_heads, d, page, block, lens, news, prefix, absent, rows_type=type, scales=scales)
    q = queries(p, heads) if q is None else q
    scale = d ** -0.5 if scale is None else scale
    got, got_lse = attend(p, heads, q, scale, window, sinks, **how)
    out, lse, size = oa.attend(*pool_values(p), p["batch"], f64(q), np.float64(np.float32(scale)), window, sinks)
    check_attend_i8(type, d, got, got_lse, out, lse, size, 2.0 ** scales[1])
    return got, got_lse


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (4, 1), (6, 2), (16, 1), (17, 1), (40, 1)])
def test_one_token_a_sequence(type, d, heads, kv_heads):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 130, 333]
    run(1, type, heads, kv_heads, d, 16, 16, lens, [1] * len(lens), uniform=True)


@pytest.mark.parametrize("page,block", [(16, 16), (32, 16), (32, 32), (64, 32), (64, 64), (128, 16), (128, 128), (256, 64), (256, 256)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (100, 4), (37, 40)])
def test_pages_blocks_and_windows_one_token(page, block, window, sinks):
    run(2, "bf16", 8, 2, 128, page, block, [600, 599, 257, 1, 40], [1] * 5, window, sinks, uniform=True)


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 2), (5, 1)])
def test_prompts(type, d, heads, kv_heads):
    run(3, type, heads, kv_heads, d, 32, 16, [150, 1, 64, 129, 33], [150, 1, 64, 129, 33])


@pytest.mark.parametrize("page,block", [(16, 16), (32, 32), (64, 16), (128, 64), (256, 256)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_pages_and_blocks_of_prompts(page, block, d):
    run(4, "bf16", 2, 1, d, page, block, [300, 70], [140, 70], 90, 20)


@pytest.mark.parametrize("news", [[1, 2, 3], [4, 1, 4], [16, 16, 15], [33, 5, 1], [70, 128, 0], [200, 0, 129]])
def test_pieces_of_prompts(news):
    run(5, "bf16", 4, 2, 128, 16, 16, [300, 200, 257], news)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (50, 3), (64, 64), (1000, 2), (2 ** 31, 0), (2 ** 32 - 1, 2 ** 32 - 1), (7, 2 ** 32 - 1)])
def test_windows_of_prompts(window, sinks):
    run(6, "f16", 2, 1, 64, 16, 16, [260, 99, 190], [260, 99, 70], window, sinks)


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2), (16, 1), (20, 1)])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("news,lens", [([150, 1], [150, 900]), ([1, 0, 2, 70, 4, 5, 16, 17, 1], [77, 30, 2, 300, 4, 500, 16, 17, 1]),
                                       ([1] * 40 + [40] + [1] * 30, [60 + 7 * i for i in range(71)])])
def test_prompts_among_single_tokens(heads, kv_heads, d, news, lens):
    """Few rows and many in one batch: each kind is a part of its own."""
    run(41, "bf16", heads, kv_heads, d, 16, 16, lens, news)
    run(42, "f16", heads, kv_heads, d, 32, 16, [n + 45 for n in lens], news, prefix=45, window=200, sinks=3)


@pytest.mark.parametrize("news,lens,kw", [([300, 1, 3], [3000, 5000, 2000], {}), ([300, 1, 3], [3000, 5000, 2000], dict(window=1000, sinks=70)),
                                          ([200, 4] * 2, [9000, 8300, 8500, 8333], dict(prefix=8192)), ([300, 1, 3], [3000, 5000, 2000], dict(max_len=1)),
                                          ([300, 1, 3], [30, 1, 2000], {}), ([40, 2, 0, 1], [50, 30000, 0, 17000], {}), ([600, 16, 1], [700, 5000, 3000], dict(absent=[(1, 3), (2, 0), (2, 40)]))])
def test_prompts_among_single_tokens_of_long_contexts(news, lens, kw):
    """Few sequences, whose keys are cut into parts for both kinds of rows; hints that are too small; sequences shorter than their rows; pages that are not there."""
    run(43, "bf16", 4, 2, 128, 32, 32, lens, news, **kw)
    # (a hint by which the few rows' keys are cut into parts of their own)
    if "prefix" not in kw:
        run(43, "bf16", 4, 2, 128, 32, 32, lens, news, **{**kw, "max_len": 2 ** 20})
        run(44, "f16", 5, 1, 256, 32, 32, lens, news, **{**kw, "max_len": 2 ** 20, "window": 0})
    run(44, "f16", 8, 1, 64, 64, 16, lens, news, **kw)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("prefix", [1, 15, 64, 100, 257])
def test_common_prefix_one_token(d, prefix):
    lens = [prefix + n for n in (1, 2, 40, 64, 65, 100, 16)]
    run(7, "bf16", 4, 2, d, 32, 16, lens, [1] * len(lens), prefix=prefix, uniform=True)


@pytest.mark.parametrize("heads,kv_heads,news", [(4, 4, [3, 1, 20]), (8, 1, [5, 30, 2]), (16, 2, [40, 40, 40])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 0), (30, 20)])
def test_common_prefix_pieces(heads, kv_heads, news, window, sinks):
    run(8, "f16", heads, kv_heads, 64, 16, 16, [170, 120, 190], news, window, sinks, prefix=75)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads", [8, 40])
def test_many_rows_behind_a_prefix(d, heads):
    run(9, "bf16", heads, 2, d, 64, 32, [300 + 3 * i for i in range(30)], [1] * 30, prefix=290, uniform=True)


def test_a_window_behind_the_prefix():
    # no row sees anything of the prefix, or only its sinks
    for sinks in (0, 5):
        run(10, "bf16", 4, 2, 64, 16, 16, [400, 390], [1, 1], window=20, sinks=sinks, prefix=200, uniform=True)


def test_rows_inside_the_prefix():
    run(11, "bf16", 2, 1, 64, 16, 16, [110, 104], [30, 4], prefix=100)


def test_absent_pages():
    away = [(0, 0), (0, 5), (0, 6), (1, 6), (2, 0), (2, 1), (2, 2), (2, 3), (3, 1)]
    run(12, "bf16", 4, 2, 128, 16, 16, [200, 100, 64, 33], [1, 1, 1, 1], absent=away, uniform=True)
    run(13, "bf16", 4, 2, 128, 16, 16, [200, 100, 64, 33], [200, 40, 64, 3], absent=away)


def test_rows_that_see_nothing():
    # lengths of zero, and sequences shorter than their rows
    run(14, "bf16", 4, 2, 64, 16, 16, [0, 3, 0, 20], [1, 1, 1, 1], uniform=True)
    run(15, "f16", 4, 2, 128, 16, 16, [0, 3, 70, 20], [2, 5, 90, 0])


@pytest.mark.parametrize("layout", ["heads first", "slice"])
def test_layouts_of_the_rows(layout):
    run(16, "bf16", 4, 2, 128, 16, 16, [100, 50], [1, 1], layout=layout, uniform=True)
    run(17, "f16", 6, 2, 64, 16, 16, [100, 50], [90, 33], layout=layout)


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales_of_the_scores(scale):
    run(18, "bf16", 4, 2, 64, 16, 16, [100, 50, 1], [1, 1, 1], scale=scale, uniform=True)
    run(19, "bf16", 4, 2, 64, 16, 16, [100, 50, 1], [60, 50, 1], scale=scale)


@pytest.mark.parametrize("scales", [(-30, 2), (-20, -18), (6, 9)])
def test_scales_of_the_blocks(scales):
    """Blocks whose scales lie far apart, and far from 1: the queries bring the scores back to ordinary ones."""
    for news in (1, 130):
        p = paged_i8(20, 2, 64, 16, 16, [140, 200], [news, news], scales=scales)
        q = (queries(p, 4).float() * 2.0 ** -(scales[1] + 4)).to(torch.bfloat16)
        got, got_lse = attend(p, 4, q, 0.5, uniform=news == 1)
        out, lse, size = oa.attend(*pool_values(p), p["batch"], f64(q), 0.5)
        check_attend_i8("bf16", 64, got, got_lse, out, lse, size, 2.0 ** scales[1])


def test_scales_that_are_no_powers_of_two():
    for news in (1, 130):
        p = paged_i8(21, 2, 128, 32, 16, [140, 200], [news, news])
        for n in ("ks", "vs"):
            p[n] = (p[n] * p["rng"].uniform(0.5, 1.0, p[n].shape)).astype(np.float32)
        q = queries(p, 4)
        got, got_lse = attend(p, 4, q, 0.1, uniform=news == 1)
        out, lse, size = oa.attend(*pool_values(p), p["batch"], f64(q), np.float64(np.float32(0.1)))
        check_attend_i8("bf16", 128, got, got_lse, out, lse, size, 2.0 ** -4)


@pytest.mark.parametrize("news", [1, 3, 70])
def test_scales_that_are_not_sound_count_as_the_smallest(news):
    """Zero, negative and NaN scales of blocks that rows see: their keys' scores and their values are 0."""
    p = paged_i8(22, 1, 64, 16, 16, [100], [news])
    pages = p["batch"]["pages"][0]
    for i, bad in enumerate((0.0, -1.0, np.nan)):
        p["ks"][pages[i]] = bad
        p["vs"][pages[i + 2]] = bad
    q = queries(p, 2)
    got, got_lse = attend(p, 2, q, 0.125, uniform=news == 1)
    k, v = pool_values(p)
    out, lse, size = oa.attend(k, v, p["batch"], f64(q), 0.125)
    check_attend_i8("bf16", 64, got, got_lse, out, lse, size, 2.0 ** -4)


@pytest.mark.parametrize("max_len", [1, 100, 5000, 2 ** 31 - 1])
def test_max_len_is_only_a_hint(max_len):
    run(23, "bf16", 4, 2, 64, 16, 16, [1500, 700], [1, 1], max_len=max_len, uniform=True)
    run(24, "bf16", 4, 2, 64, 16, 16, [300, 100], [100, 70], max_len=max_len, prefix=30)


@pytest.mark.parametrize("news", [1, 40])
def test_growing_scores(news):
    """Scores that rise along the keys by far more than the range of a weight: the maximum moves all the time."""
    p = paged_i8(25, 1, 64, 16, 16, [700], [news])
    q = torch.ones((news, 2, 64), dtype=torch.bfloat16)
    for sign in (1, -1):
        for j in range(700):
            pg, at = oa.place_of(p["batch"], 0, j, 16, p["n_pages"])
            p["k"][pg, :, at] = sign * (j % 16 + 1)
            p["ks"][pg] = 1.0 + j // 16
        got, got_lse = attend(p, 2, q, 0.25, uniform=news == 1)
        out, lse, size = oa.attend(*pool_values(p), p["batch"], f64(q), 0.25)
        check_attend_i8("bf16", 64, got, got_lse, out, lse, size, 2.0 ** -4)


@pytest.mark.parametrize("news", [1, 30])
def test_many_small_weights_beside_a_large_one(news):
    """One key far above 3000 others whose weights together count."""
    p = paged_i8(26, 1, 64, 64, 64, [3001], [news], rows_type="f16")
    q = torch.ones((news, 1, 64), dtype=torch.float16)
    p["k"][:] = 0
    pg, at = oa.place_of(p["batch"], 0, 5, 64, p["n_pages"])
    p["k"][pg, :, at] = 80
    p["ks"][:] = np.where(np.isfinite(p["ks"]) & (p["ks"] > 0), 2.0 ** -8, p["ks"])
    got, got_lse = attend(p, 1, q, 0.85, uniform=news == 1)
    out, lse, size = oa.attend(*pool_values(p), p["batch"], f64(q), np.float64(np.float32(0.85)))
    check_attend_i8("f16", 64, got, got_lse, out, lse, size, 2.0 ** -4)


def test_queries_that_are_no_numbers_reach_only_their_rows():
    for news in (130, 2):
        p = paged_i8(27, 1, 64, 16, 16, [140], [news])
        q = queries(p, 2)
        q[-1, 0, 3] = float("nan")
        got, got_lse = attend(p, 2, q, 0.125)
        clean = q.clone()
        clean[-1, 0, 3] = 0
        out, lse, size = oa.attend(*pool_values(p), p["batch"], f64(clean), 0.125)
        assert np.isnan(got[-1, 0]).all() and np.isnan(got_lse[-1, 0])
        got[-1, 0], got_lse[-1, 0] = out[-1, 0], lse[-1, 0]
        check_attend_i8("bf16", 64, got, got_lse, out, lse, size, 2.0 ** -4)


@pytest.mark.parametrize("news", [1, 20, 130])
@pytest.mark.parametrize("power", [-126, -100, -30, 30, 100, 120])
def test_queries_of_any_size(news, power):
    """Queries far from 1, rows of very different sizes, and a scale that makes ordinary scores of the largest ones."""
    p = paged_i8(38, 2, 128, 16, 16, [200, 140], [news, news])
    q = queries(p, 4).float()
    q = (q * 2.0 ** power).to(torch.bfloat16)
    q[::3, 1] = (q[::3, 1].float() * 2.0 ** -20).to(torch.bfloat16)
    q[0, 0] = 0
    scale = 2.0 ** -power * 0.1
    got, got_lse = attend(p, 4, q, scale, uniform=news == 1)
    out, lse, size = oa.attend(*pool_values(p), p["batch"], f64(q), np.float64(np.float32(scale)))
    check_attend_i8("bf16", 128, got, got_lse, out, lse, size, 2.0 ** -4)


@pytest.mark.parametrize("news", [1, 130])
def test_keys_of_large_and_small_scales(news):
    """Scales of the keys far from 1, with a scale of the scores that brings them back: no product on the way leaves the range."""
    for power in (-110, 110):
        p = paged_i8(39, 1, 64, 16, 16, [150], [news])
        p["ks"] = np.where(np.isfinite(p["ks"]) & (p["ks"] > 0) & (p["ks"] < 1), p["ks"] * np.float32(2.0 ** power), p["ks"]).astype(np.float32)
        q = queries(p, 2)
        scale = 0.125 * 2.0 ** -power
        got, got_lse = attend(p, 2, q, scale, uniform=news == 1)
        out, lse, size = oa.attend(*pool_values(p), p["batch"], f64(q), np.float64(np.float32(scale)))
        check_attend_i8("bf16", 64, got, got_lse, out, lse, size, 2.0 ** -4)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("news,window,sinks", [(1, 100, 0), (20, 300, 5), (200, 64, 0), (300, 1, 20)])
def test_the_last_positions_there_are(d, news, window, sinks):
    """A sequence that ends at the last position, through a window; all pages but the first and the last ones have been given back."""
    print(f"case i8 last positions d={d} news={news} window={window} sinks={sinks}", flush=True)
    most, page, kept = 2 ** 31 - 2 ** 16, 256, 3
    stride = most // page
    p = paged_i8(40, 1, d, page, 64, [(kept + 1) * page], [news])
    order = p["batch"]["pages"][0]
    q = queries(p, 2)
    table = torch.full((1, stride), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = int(order[0])
    table[0, -kept:] = torch.from_numpy(order[1:].copy()).cuda()
    cache, t = device_cache_i8(p)
    starts, lens = torch.tensor([0, news], dtype=torch.int32, device="cuda"), torch.tensor([most], dtype=torch.int32, device="cuda")
    batch = dc.KVBatch(1, news, news, most, lens, table, stride, row_start_dev=starts)
    qd = q.cuda()
    out, lse = torch.empty_like(qd), torch.empty((news, 2), dtype=torch.float32, device="cuda")
    a = dc.Attention(2, qd, out, lse, d ** -0.5, window=window, sinks=sinks)
    n = dc.attention_paged_workspace(cache, batch, a)
    ws = torch.empty(n + 16, dtype=torch.uint8, device="cuda")
    dc.attention_paged(cache, batch, a, ws, n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    # the same rows in a sequence without the pages between
    want = oa.attend(*pool_values(p), p["batch"], f64(q), np.float64(np.float32(d ** -0.5)), window, sinks)
    check_attend_i8("bf16", d, f64(out), f64(lse), *want, 2.0 ** -4)


def test_lse_may_be_left_out_and_results_repeat():
    for news, prefix in ((1, 0), (1, 64), (150, 0)):
        p = paged_i8(28, 2, 128, 16, 16, [900, 300], [news, news], prefix)
        q = queries(p, 8).cuda()
        cache, t = device_cache_i8(p)
        batch = device_batch(p)
        results = []
        for with_lse in (True, False, True):
            out = torch.empty_like(q)
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda") if with_lse else None
            a = dc.Attention(8, q, out, lse, 0.1)
            n = dc.attention_paged_workspace(cache, batch, a)
            ws = torch.full((n + 16,), 0xA5, dtype=torch.uint8, device="cuda")
            dc.attention_paged(cache, batch, a, ws, n, torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            results.append(out.view(torch.int16).cpu())
        assert torch.equal(results[0], results[1]) and torch.equal(results[0], results[2])


def test_another_stream():
    s = torch.cuda.Stream()
    run(29, "bf16", 8, 2, 128, 32, 32, [500, 400, 77], [1, 1, 1], stream=s, uniform=True)
    run(30, "bf16", 8, 2, 128, 32, 32, [500, 400, 77], [300, 1, 77], stream=s, prefix=40)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_long_contexts(d):
    """Runs of keys that are cut and joined, of one sequence and of several."""
    run(31, "bf16", 8, 1, d, 128, 64, [9001], [1], uniform=True)
    run(32, "bf16", 4, 2, d, 32, 16, [3001, 17, 1500], [1, 1, 1], uniform=True)
    run(33, "f16", 4, 1, d, 64, 32, [4000], [7])
    run(34, "f16", 4, 1, d, 64, 32, [2500, 600], [40, 3])


@pytest.mark.parametrize("heads,kv_heads,d,lens,news", [(16, 2, 64, [6000], [300]), (12, 4, 128, [3000], [400]), (5, 1, 256, [2000, 1990], [100, 90]), (20, 5, 64, [700] * 30, [1] * 30)])
def test_parts_of_many_rows(heads, kv_heads, d, lens, news):
    """Keys in parts, whose results are joined for many rows and heads."""
    run(45, "bf16", heads, kv_heads, d, 64, 64, lens, news, uniform=max(news) == 1)
    run(46, "f16", heads, kv_heads, d, 64, 32, lens, news, window=900, sinks=2, absent=[(0, 1)], uniform=max(news) == 1)


@pytest.mark.parametrize("lens,news,prefix", [([300, 70, 900], [150, 1, 2], 0), ([2500, 1800], [300, 1], 0), ([1900] * 40, [1] * 40, 1024), ([900, 800, 850], [60, 3, 40], 700), ([50, 60], [1, 2], 0)])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_behind_the_last_sequence(lens, news, prefix, d):
    """Rows of no sequence, as a recorded step has them: their results stay as they were."""
    print(f"case i8 rows behind lens={lens} news={news} prefix={prefix} d={d}", flush=True)
    p = paged_i8(47, 2, d, 32, 32, lens, news, prefix)
    heads, rows, more = 8, int(p["batch"]["starts"][-1]), 150
    q = queries(p, heads)
    cache, t = device_cache_i8(p)
    starts = torch.from_numpy(p["batch"]["starts"]).cuda()
    lens_d, pages = torch.from_numpy(p["batch"]["lens"]).cuda(), torch.from_numpy(p["batch"]["pages"]).cuda()
    prefix_pages = torch.from_numpy(p["batch"]["prefix_pages"]).cuda()
    b = dc.KVBatch(len(lens), rows + more, max(news), max(lens), lens_d, pages, pages.shape[1], row_start_dev=starts, prefix_len=prefix,
                   prefix_pages_dev=prefix_pages if prefix else None)
    qd = torch.full((rows + more, heads, d), float("nan"), dtype=q.dtype, device="cuda")
    qd[:rows] = q.cuda()
    out = torch.full_like(qd, SENTINEL)
    lse = torch.full((rows + more, heads), SENTINEL, dtype=torch.float32, device="cuda")
    a = dc.Attention(heads, qd, out, lse, d ** -0.5)
    n = dc.attention_paged_workspace(cache, b, a)
    ws = torch.full((n + 16,), 0xFF, dtype=torch.uint8, device="cuda")
    dc.attention_paged(cache, b, a, ws, n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (out[rows:] == SENTINEL).all() and (lse[rows:] == SENTINEL).all()
    want = oa.attend(*pool_values(p), p["batch"], f64(q), np.float64(np.float32(d ** -0.5)))
    check_attend_i8("bf16", d, f64(out[:rows]), f64(lse[:rows]), *want, 2.0 ** -4)


def test_pools_of_more_than_four_gib():
    """Pages beyond 2^32 bytes of the pools."""
    d, page, kv, block = 128, 256, 8, 32
    n_pages = (5 << 30) // (page * kv * d)
    print(f"case attention i8 pool of {n_pages} pages", flush=True)
    p = paged_i8(35, kv, d, page, block, [700, 300], [1, 30])
    far = n_pages - p["n_pages"]
    pools = [torch.zeros((n_pages, kv, page, d), dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.full((n_pages, kv, page // block), float("nan"), device="cuda") for _ in range(2)]
    for big, small in zip(pools + scales, ("k", "v", "ks", "vs")):
        big[far:] = torch.from_numpy(p[small]).cuda()
    q = queries(p, kv)
    table = torch.from_numpy(np.where(p["batch"]["pages"] >= 0, p["batch"]["pages"] + far, -1).astype(np.int32)).cuda()
    lens, starts = torch.from_numpy(p["batch"]["lens"]).cuda(), torch.from_numpy(p["batch"]["starts"]).cuda()
    cache = dc.KVCache(pools[0], pools[1], n_pages, kv, d, page, dc.TYPE_I8, scale_tokens=block, k_scale_dev=scales[0], v_scale_dev=scales[1])
    qd, out = q.cuda(), torch.empty(q.shape, dtype=q.dtype, device="cuda")
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    for lo, hi in ((0, 1), (0, 2)):
        batch = dc.KVBatch(hi, int(starts[hi]), 30 if hi == 2 else 1, 700, lens, table, table.shape[1], row_start_dev=starts)
        a = dc.Attention(kv, qd, out, lse, 0.1)
        n = dc.attention_paged_workspace(cache, batch, a)
        ws = torch.empty(n + 16, dtype=torch.uint8, device="cuda")
        dc.attention_paged(cache, batch, a, ws, n, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        rows = int(starts[hi])
        ref, ref_lse, size = oa.attend(*pool_values(p), p["batch"], f64(q), np.float64(np.float32(0.1)))
        check_attend_i8("bf16", d, f64(out)[:rows], f64(lse)[:rows], ref[:rows], ref_lse[:rows], {n: s[:rows] for n, s in size.items()}, 2.0 ** -4)


def test_replays_of_a_recorded_call():
    for news, prefix in ((1, 0), (1, 200), (150, 30)):
        p = paged_i8(36, 2, 128, 16, 16, [900, 300], [news, news], prefix)
        q = queries(p, 8).cuda()
        cache, t = device_cache_i8(p)
        batch = device_batch(p)
        out = torch.empty_like(q)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
        a = dc.Attention(8, q, out, lse, 0.1)
        n = dc.attention_paged_workspace(cache, batch, a)
        ws = torch.empty(n + 16, dtype=torch.uint8, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        dc.attention_paged(cache, batch, a, ws, n, side.cuda_stream)
        torch.cuda.synchronize()
        want = out.view(torch.int16).cpu().clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            dc.attention_paged(cache, batch, a, ws, n, side.cuda_stream)
        for _ in range(4):
            out.zero_()
            ws.fill_(0x5A)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16).cpu(), want)


def test_device_arrays_that_do_not_fit_are_survived():
    """Rows, lengths and pages outside what the call was told of: the rows of the other sequences are right, nothing outside is written."""
    p = paged_i8(37, 2, 64, 16, 16, [100, 60, 30], [1, 1, 1])
    q = queries(p, 4)
    want, want_lse = attend(p, 4, q, 0.125, uniform=True)
    for lens in ([100, 60, 2 ** 31 - 1], [100, 60, -5], [100, 60, 31 + 16 * 7]):
        other = dict(p, batch=dict(p["batch"], lens=np.array(lens, dtype=np.int32)))
        got, got_lse = attend(other, 4, q, 0.125, uniform=True)
        assert np.array_equal(got[:2], want[:2]) and np.array_equal(got_lse[:2], want_lse[:2])
    for starts in ([0, 1, 2, 2 ** 31 - 1], [0, 1, 2, -7], [0, 1, 2, 2], [-3, 1, 2, 3]):
        other = dict(p, batch=dict(p["batch"], starts=np.array(starts, dtype=np.int32)))
        cache, t = device_cache_i8(p)
        dev = {n: torch.from_numpy(np.ascontiguousarray(other["batch"][n])).cuda() for n in ("lens", "starts", "pages")}
        batch = dc.KVBatch(3, 3, 3, 100, dev["lens"], dev["pages"], p["batch"]["pages"].shape[1], row_start_dev=dev["starts"])
        out = torch.full((5, 4, 64), SENTINEL, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((5, 4), SENTINEL, dtype=torch.float32, device="cuda")
        qd = q.cuda()
        a = dc.Attention(4, qd, out[1:-1], lse[1:-1], 0.125)
        n = dc.attention_paged_workspace(cache, batch, a)
        ws = torch.empty(n + 16, dtype=torch.uint8, device="cuda")
        dc.attention_paged(cache, batch, a, ws, n, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert (out[0] == SENTINEL).all() and (out[-1] == SENTINEL).all()
        assert np.array_equal(f64(out[2]), want[1])
