"""dc_attention_paged against the oracle in 64 bits through the C ABI: types, head sizes and groups, lengths from nothing to several
tiles, windows and sinks, absent pages, common prefixes, layouts of the rows, and what must have no influence (every value of the
pools that belongs to no token is NaN)."""
import numpy as np
import pytest

import oracle.attention as oa
import paper_2502_15443_amd as dc
from tests.attention_cases import KIND, check_attend, device_batch, device_cache, f64, paged, rows_tensor, torch_type

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SENTINEL = 7.75


def attend(p, heads, q, scale, window=0, sinks=0, layout="dense", uniform=False, max_len=None, stream=None, extra_rows=0):
    """(out, lse) as fp64 arrays; checks that nothing outside the rows was written."""
    cache, k, v = device_cache(p)
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
    assert torch.equal(k.cpu().view(torch.int16), p["k"].view(torch.int16))
    return f64(out), f64(lse[1:-1])


def queries(p, heads, type):
    rows = int(p["batch"]["starts"][-1])
    return torch.from_numpy(p["rng"].standard_normal((rows, heads, p["head_dim"])).astype(np.float32) * 1.5).to(torch_type(type))


def run(seed, type, heads, kv_heads, d, page, lens, news, window=0, sinks=0, prefix=0, absent=(), scale=None, **how):
    print(f"case attention {type} heads={heads}/{kv_heads} d={d} page={page} lens={lens} news={news} window={window} sinks={sinks} "
          f"prefix={prefix} absent={absent} {how}", flush=True)
    p = paged(seed, type, kv_heads, d, page, lens, news, prefix, absent)
    q = queries(p, heads, type)
    scale = d ** -0.5 if scale is None else scale
    got, got_lse = attend(p, heads, q, scale, window, sinks, **how)
    out, lse, size = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q), np.float64(np.float32(scale)), window, sinks)
    check_attend(type, d, got, got_lse, out, lse, size)
    return got, got_lse


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (4, 1), (6, 2), (16, 1), (17, 1), (40, 1)])
def test_one_token_a_sequence(type, d, heads, kv_heads):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 130, 333]
    run(1, type, heads, kv_heads, d, 16, lens, [1] * len(lens), uniform=True)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (100, 4), (37, 40)])
def test_pages_and_windows_one_token(page, window, sinks):
    run(2, "bf16", 8, 2, 128, page, [600, 599, 257, 1, 40], [1] * 5, window, sinks, uniform=True)


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 2), (5, 1)])
def test_prompts(type, d, heads, kv_heads):
    run(3, type, heads, kv_heads, d, 32, [150, 1, 64, 129, 33], [150, 1, 64, 129, 33])


@pytest.mark.parametrize("news", [[1, 2, 3], [4, 1, 4], [16, 16, 15], [33, 5, 1], [70, 128, 0], [200, 0, 129]])
def test_pieces_of_prompts(news):
    run(4, "bf16", 4, 2, 128, 16, [300, 200, 257], news)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (50, 3), (64, 64), (1000, 2), (2 ** 31, 0), (2 ** 32 - 1, 2 ** 32 - 1), (7, 2 ** 32 - 1)])
def test_windows_of_prompts(window, sinks):
    run(5, "f16", 2, 1, 64, 16, [260, 99, 190], [260, 99, 70], window, sinks)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("prefix", [1, 15, 64, 100, 257])
def test_common_prefix_one_token(d, prefix):
    lens = [prefix + n for n in (1, 2, 40, 64, 65, 100, 16)]
    run(6, "bf16", 4, 2, d, 32, lens, [1] * len(lens), prefix=prefix, uniform=True)


@pytest.mark.parametrize("heads,kv_heads,news", [(4, 4, [3, 1, 20]), (8, 1, [5, 30, 2]), (16, 2, [40, 40, 40])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 0), (30, 20)])
def test_common_prefix_pieces(heads, kv_heads, news, window, sinks):
    run(7, "f16", heads, kv_heads, 64, 16, [170, 120, 190], news, window, sinks, prefix=75)


def test_many_rows_behind_a_prefix():
    run(8, "bf16", 8, 2, 128, 64, [300 + 3 * i for i in range(70)], [1] * 70, prefix=290, uniform=True)


def test_a_window_behind_the_prefix():
    # no row sees anything of the prefix, or only its sinks
    for sinks in (0, 5):
        run(9, "bf16", 4, 2, 64, 16, [400, 390], [1, 1], window=20, sinks=sinks, prefix=200, uniform=True)


def test_rows_inside_the_prefix():
    # more rows than tokens behind the prefix: the first rows lie in the prefix, whose later tokens they must not see
    run(10, "bf16", 2, 1, 64, 16, [110, 104], [30, 4], prefix=100)


def test_absent_pages():
    run(11, "bf16", 4, 2, 128, 16, [200, 100, 64, 33], [1, 1, 1, 1], absent=[(0, 0), (0, 5), (0, 6), (1, 6), (2, 0), (2, 1), (2, 2), (2, 3), (3, 1)], uniform=True)
    run(12, "bf16", 4, 2, 128, 16, [200, 100, 64, 33], [200, 40, 64, 3], absent=[(0, 0), (0, 5), (0, 6), (1, 6), (2, 0), (2, 1), (2, 2), (2, 3), (3, 1)])


def test_rows_that_see_nothing():
    # lengths of zero, and sequences shorter than their rows
    run(13, "bf16", 4, 2, 64, 16, [0, 3, 0, 20], [1, 1, 1, 1], uniform=True)
    run(14, "f16", 4, 2, 128, 16, [0, 3, 70, 20], [2, 5, 90, 0])


@pytest.mark.parametrize("layout", ["heads first", "slice"])
def test_layouts_of_the_rows(layout):
    run(15, "bf16", 4, 2, 128, 16, [100, 50], [1, 1], layout=layout, uniform=True)
    run(16, "f16", 6, 2, 64, 16, [100, 50], [90, 33], layout=layout)


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(scale):
    run(17, "bf16", 4, 2, 64, 16, [100, 50, 1], [1, 1, 1], scale=scale, uniform=True)
    run(18, "bf16", 4, 2, 64, 16, [100, 50, 1], [60, 50, 1], scale=scale)


@pytest.mark.parametrize("max_len", [1, 100, 5000, 2 ** 31 - 1])
def test_max_len_is_only_a_hint(max_len):
    run(19, "bf16", 4, 2, 64, 16, [1500, 700], [1, 1], max_len=max_len, uniform=True)
    run(20, "bf16", 4, 2, 64, 16, [300, 100], [100, 70], max_len=max_len, prefix=30)


@pytest.mark.parametrize("news", [1, 40])
def test_growing_scores(news):
    """Scores that rise along the keys by far more than the range of a weight: the maximum moves all the time."""
    p = paged(21, "bf16", 1, 64, 16, [700], [news])
    q = torch.ones((news, 2, 64), dtype=torch.bfloat16)
    ramp = torch.arange(p["n_pages"] * 16, dtype=torch.float32)
    for sign in (1, -1):
        for j in range(700):
            pg, at = oa.place_of(p["batch"], 0, j, 16, p["n_pages"])
            p["k"][pg, :, at] = sign * float(ramp[j]) / 8
        got, got_lse = attend(p, 2, q, 1.0, uniform=news == 1)
        out, lse, size = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q), 1.0)
        check_attend("bf16", 64, got, got_lse, out, lse, size)


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 8)])
@pytest.mark.parametrize("news", [130, 3])
def test_values_that_are_no_numbers_reach_only_the_rows_that_see_them(type, value, window, sinks, news):
    print(f"case attention not finite {type} {value} window={window} sinks={sinks} news={news}", flush=True)
    p = paged(22, type, 2, 128, 16, [140], [news])
    q = queries(p, 4, type)
    bad = [3, 60, 139 - news // 2, 138]
    for n, j in enumerate(bad):
        pg, at = oa.place_of(p["batch"], 0, j, 16, p["n_pages"])
        p["v"][pg, n % 2, at, 7 * n] = value
    got, got_lse = attend(p, 4, q, 128 ** -0.5, window, sinks)
    clean = {k: v for k, v in p.items()}
    clean["v"] = p["v"].nan_to_num(0.0, 0.0, 0.0)
    out, lse, size = oa.attend(f64(clean["k"]), f64(clean["v"]), p["batch"], f64(q), np.float64(np.float32(128 ** -0.5)), window, sinks)
    mark = np.zeros(out.shape, dtype=bool)  # results that see such a value
    for n, j in enumerate(bad):
        for row in range(news):
            pos = 140 - news + row
            if j <= pos and (not window or j > pos - window or j < sinks):
                mark[row, 2 * (n % 2):2 * (n % 2) + 2, 7 * n] = True
    assert mark.any() and not mark.all()
    assert not np.isfinite(got[mark]).any()
    if np.isnan(value):
        assert np.isnan(got[mark]).all()
    elif type == "bf16":
        assert (got[mark] == value).all()
    check_attend(type, 128, np.where(mark, out, got), got_lse, out, lse, size)


def test_keys_that_are_no_numbers_reach_only_the_rows_that_see_them():
    for news in (130, 2):
        p = paged(23, "bf16", 1, 64, 16, [140], [news])
        q = queries(p, 2, "bf16")
        pg, at = oa.place_of(p["batch"], 0, 139, 16, p["n_pages"])
        p["k"][pg, 0, at, 5] = float("nan")
        got, got_lse = attend(p, 2, q, 0.125)
        out, lse, size = oa.attend(f64(p["k"].nan_to_num(0.0)), f64(p["v"]), p["batch"], f64(q), 0.125)
        assert np.isnan(got[-1]).all() and np.isnan(got_lse[-1]).all()
        check_attend("bf16", 64, got[:-1], got_lse[:-1], out[:-1], lse[:-1], {k: v[:-1] for k, v in size.items()})


def test_lse_may_be_left_out_and_results_repeat():
    for news, prefix in ((1, 0), (1, 64), (150, 0)):
        p = paged(24, "bf16", 2, 128, 16, [900, 300], [news, news], prefix)
        q = queries(p, 8, "bf16").cuda()
        cache, k, v = device_cache(p)
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
    run(25, "bf16", 8, 2, 128, 32, [500, 400, 77], [1, 1, 1], stream=s, uniform=True)
    run(26, "bf16", 8, 2, 128, 32, [500, 400, 77], [300, 1, 77], stream=s, prefix=40)


def test_a_pool_of_more_than_four_gib():
    """Pages beyond 2^32 bytes and 2^31 elements of the pools."""
    d, page, kv = 128, 256, 8
    n_pages = (5 << 30) // (page * kv * d * 2)
    print(f"case attention pool of {n_pages} pages", flush=True)
    p = paged(27, "bf16", kv, d, page, [700, 300], [1, 30])
    k = torch.zeros((n_pages, kv, page, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    far = n_pages - p["n_pages"]
    k[far:], v[far:] = p["k"].cuda(), p["v"].cuda()
    q = queries(p, kv, "bf16")
    table = torch.from_numpy(np.where(p["batch"]["pages"] >= 0, p["batch"]["pages"] + far, -1).astype(np.int32)).cuda()
    lens, starts = torch.from_numpy(p["batch"]["lens"]).cuda(), torch.from_numpy(p["batch"]["starts"]).cuda()
    cache = dc.KVCache(k, v, n_pages, kv, d, page, KIND["bf16"])
    qd, out = q.cuda(), torch.empty(q.shape, dtype=q.dtype, device="cuda")
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    for lo, hi in ((0, 1), (0, 2)):
        batch = dc.KVBatch(hi, int(starts[hi]), 30 if hi == 2 else 1, 700, lens, table, table.shape[1], row_start_dev=starts)
        a = dc.Attention(kv, qd, out, lse, 0.1)
        n = dc.attention_paged_workspace(cache, batch, a)
        ws = torch.empty(n + 16, dtype=torch.uint8, device="cuda")
        dc.attention_paged(cache, batch, a, ws, n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    ref, ref_lse, size = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q), np.float64(np.float32(0.1)))
    check_attend("bf16", d, f64(out), f64(lse), ref, ref_lse, size)


def test_replays_of_a_recorded_call():
    for news, prefix in ((1, 0), (1, 200), (150, 30)):
        p = paged(28, "bf16", 2, 128, 16, [900, 300], [news, news], prefix)
        q = queries(p, 8, "bf16").cuda()
        cache, k, v = device_cache(p)
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
    p = paged(29, "bf16", 2, 64, 16, [100, 60, 30], [1, 1, 1])
    q = queries(p, 4, "bf16")
    want, want_lse = attend(p, 4, q, 0.125, uniform=True)
    for lens in ([100, 60, 2 ** 31 - 1], [100, 60, -5], [100, 60, 31 + 16 * 7]):
        other = dict(p, batch=dict(p["batch"], lens=np.array(lens, dtype=np.int32)))
        got, got_lse = attend(other, 4, q, 0.125, uniform=True)
        assert np.array_equal(got[:2], want[:2]) and np.array_equal(got_lse[:2], want_lse[:2])
    for starts in ([0, 1, 2, 2 ** 31 - 1], [0, 1, 2, -7], [0, 1, 2, 2], [-3, 1, 2, 3]):
        other = dict(p, batch=dict(p["batch"], starts=np.array(starts, dtype=np.int32)))
        cache, k, v = device_cache(p)
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
