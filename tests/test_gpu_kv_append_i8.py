"""dc_kv_append into a cache of 8 bits against the oracle through the C ABI: whole numbers, scales and turned queries are the same bits; types, pairings,
blocks and pages, pieces that begin inside a block, scales that grow, values that are no numbers, and everything that must stay as it was."""
import numpy as np
import pytest

import oracle.cache_i8 as oc8
import paper_2502_15443_amd as dc
from tests.attention_cases import KIND, device_batch, rows_tensor, torch_type
from tests.i8_cases import device_cache_i8, paged_i8
from tests.test_cache_alignment import _rows_at
from tests.test_gpu_kv_append import angles

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SENTINEL = 7.75


def rows_of(p, x_type, heads, spread=3):
    """New rows whose magnitudes differ by powers of two from row to row and head to head."""
    rows = int(p["batch"]["starts"][-1])
    r = p["rng"]
    return {n: torch.from_numpy((r.standard_normal((rows, h, p["head_dim"])) * 2.0 ** r.integers(-spread, spread + 1, (rows, h, 1))).astype(np.float32))
            .to(torch_type(x_type)) for n, h in (("k", p["kv_heads"]), ("v", p["kv_heads"]), ("q", heads))}


def check(p, x, t, out, cos, sin, neighbours, positions=None, max_new=None, wide=None):
    want = oc8.append(p["k"], p["v"], p["ks"], p["vs"], p["batch"], p["block"], x["k"].float().numpy(), x["v"].float().numpy(), cos, sin, neighbours,
                      positions, max_new)
    for got, w, what in zip(t, want, ("k", "v", "k scale", "v scale")):
        g = got.cpu().numpy()
        g, w = (g.view(np.uint32), w.view(np.uint32)) if g.dtype == np.float32 else (g, w)
        assert np.array_equal(g, w), (what, int((g != w).sum()), np.argwhere(g != w)[:3].tolist())
    if out is None:
        return
    b, xq = p["batch"], x["q"].float().numpy()
    got = out.cpu()
    for s, length in enumerate(b["lens"]):
        first, end = int(b["starts"][s]), int(b["starts"][s + 1])
        for row in range(first, end):
            at = int(length) - (end - row) if positions is None else int(positions[row])
            left = (cos.shape[1] and not 0 <= at < len(cos)) or (max_new is not None and row - first >= max_new)
            w = np.full(xq[row].shape, SENTINEL) if left else oc8.rotate32(xq[row], cos[at], sin[at], neighbours) if cos.shape[1] else xq[row]
            assert torch.equal(got[row], torch.from_numpy(w.astype(np.float32)).to(got.dtype)), row
    if wide is not None:
        edge = wide.clone()
        edge[1:-1, 1:-1] = SENTINEL
        assert (edge == SENTINEL).all()


def run(seed, rows_type, x_type, heads, kv_heads, d, page, block, lens, news, rot, neighbours=False, prefix=0, absent=(), layout="dense", positions=None,
        n_positions=None, uniform=False, stream=None, x=None, scales=(-6, -4), max_new=None):
    print(f"case append i8 {x_type}->{rows_type} heads={heads}/{kv_heads} d={d} page={page} block={block} lens={lens} news={news} rot={rot} "
          f"neighbours={neighbours} prefix={prefix} layout={layout}", flush=True)
    p = paged_i8(seed, kv_heads, d, page, block, lens, news, prefix, absent, rows_type=rows_type, scales=scales)
    x = rows_of(p, x_type, heads) if x is None else x
    n_positions = n_positions or max(lens)
    cos, sin = angles(n_positions, rot // 2)
    cache, t = device_cache_i8(p)
    batch = device_batch(p, uniform)
    if max_new:
        batch.max_new = max_new
    kd, vd, qd = (rows_tensor(x[n].cuda(), layout) if x[n].shape[1] else None for n in ("k", "v", "q"))
    rows = x["k"].shape[0]
    wide = torch.full((rows + 2, heads + 2, d), SENTINEL, dtype=torch_type(rows_type), device="cuda")
    out = wide[1:-1, 1:-1] if heads else None
    pos_d = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda")
    cd, sd = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    r = dc.KVRows(KIND[x_type], heads, kd, vd, qd, out, rot_dim=rot, pairing=int(neighbours), cos_dev=cd if rot else None, sin_dev=sd if rot else None,
                  n_positions=n_positions, position_dev=pos_d)
    torch.cuda.synchronize()
    dc.kv_append(cache, batch, r, torch.cuda.current_stream().cuda_stream if stream is None else stream.cuda_stream)
    torch.cuda.synchronize()
    check(p, x, t, out, cos, sin, neighbours, positions, max_new, wide if heads else None)
    return p, x, t


@pytest.mark.parametrize("rows_type", ["bf16", "f16"])
@pytest.mark.parametrize("x_type", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("neighbours", [False, True])
def test_types_and_pairings(rows_type, x_type, d, neighbours):
    run(1, rows_type, x_type, 6, 2, d, 32, 16, [40, 1, 33], [40, 1, 2], d, neighbours)


@pytest.mark.parametrize("page,block", [(16, 16), (32, 16), (32, 32), (64, 16), (64, 64), (128, 32), (128, 128), (256, 16), (256, 64), (256, 256)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_pages_and_blocks(page, block, d):
    # whole pieces, pieces from inside a block, single tokens at a block's end, its beginning and its second place
    run(2, "bf16", "f32", 2, 1, d, page, block, [300, 290, block, block + 1, block + 2, 70], [300, 150, 1, 1, 1, 30], d)


@pytest.mark.parametrize("new", [1, 2, 3, 4, 5, 6, 15, 16, 17, 33])
@pytest.mark.parametrize("d,kv_heads", [(64, 5), (128, 3)])
def test_few_and_many_new_tokens(new, d, kv_heads):
    lens = [new + n for n in (0, 1, 7, 13, 15, 16, 30)]
    run(3, "f16", "bf16", 3, kv_heads, d, 32, 16, lens, [new] * len(lens), d // 2, True)


@pytest.mark.parametrize("rot", [0, 16, 48, 64, 112, 128])
@pytest.mark.parametrize("neighbours", [False, True])
def test_partial_rotation(rot, neighbours):
    run(4, "bf16", "f32", 5, 5, 128, 16, 16, [30, 17], [7, 17], rot, neighbours)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (32, 32), (40, 40), (64, 8), (71, 1), (0, 4)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_heads(heads, kv_heads, d):
    run(5, "bf16", "bf16", heads, kv_heads, d, 64, 32, [100, 3, 65], [1, 1, 1], d, uniform=True)
    run(6, "bf16", "bf16", heads, kv_heads, d, 64, 32, [40, 30], [12, 1], d)


@pytest.mark.parametrize("layout", ["heads first", "slice"])
def test_layouts(layout):
    run(7, "f16", "f16", 6, 2, 128, 16, 16, [60, 31], [60, 5], 128, True, layout=layout)


def test_many_rows():
    # more rows than a launch of few rows has; sequences without rows among them; more sequences than a wavefront has lanes
    run(8, "bf16", "bf16", 4, 2, 64, 16, 16, [300, 0, 290, 7], [300, 0, 280, 0], 64)
    run(9, "bf16", "bf16", 2, 1, 64, 32, 16, [1 + i % 41 for i in range(150)], [min(1 + i % 41, i % 9) for i in range(150)], 64)
    # a prompt among single tokens
    run(10, "bf16", "bf16", 2, 1, 64, 32, 32, [20 + i for i in range(70)] + [200] + [5] * 10, [1] * 70 + [170] + [1] * 10, 64)


def test_rows_of_every_kind_of_launch():
    # many single tokens, of few and of many heads
    run(30, "bf16", "bf16", 2, 1, 64, 16, 16, [1 + i % 37 for i in range(700)], [1] * 700, 64, uniform=True)
    run(31, "f16", "f32", 33, 3, 64, 16, 16, [2 + i % 37 for i in range(600)], [2] * 600, 32)
    # many rows of many query heads: queries apart from the rest, single tokens between
    run(32, "bf16", "bf16", 64, 1, 64, 32, 32, [2100, 40, 1999], [2100, 1, 1999], 64)


def test_prefix_and_absent_pages():
    run(11, "bf16", "f32", 4, 2, 64, 16, 16, [130, 100, 75], [20, 25, 1], 32, prefix=70, absent=[(0, 1), (1, 1)])
    # rows that begin inside the prefix: its last block ends with it, and the own pages begin with a block
    run(12, "bf16", "f32", 2, 1, 64, 16, 16, [110], [40], 64, prefix=75)
    run(13, "bf16", "f32", 2, 1, 64, 32, 32, [80, 78], [6, 1], 64, prefix=77)


def test_rows_without_a_place():
    # sequences shorter than their rows: positions below zero have no cosines, nothing is written for them
    run(14, "bf16", "bf16", 4, 2, 64, 16, 16, [3, 0, 20], [5, 1, 2], 64)
    run(15, "bf16", "bf16", 4, 2, 64, 16, 16, [3, 0, 20], [9, 1, 2], 0)


def test_given_positions():
    # rows whose cosines are not in the table are left out as a whole: they count for no scale
    run(16, "bf16", "bf16", 4, 2, 64, 16, 16, [10, 20], [3, 4], 64, positions=[0, 5, 2, 99, 100, -1, 50], n_positions=100)
    run(17, "bf16", "bf16", 4, 2, 64, 16, 16, [20, 30], [18, 12], 64, positions=[7] * 3 + [200] + [9] * 14 + [100] * 12, n_positions=100)


def test_rows_beyond_max_new():
    run(18, "bf16", "bf16", 2, 2, 64, 16, 16, [60, 40], [30, 3], 64, max_new=20)
    run(19, "bf16", "bf16", 2, 2, 64, 16, 16, [60, 40], [7, 3], 64, max_new=2)


@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("scales", [(-40, -38), (-2, 8), (-126, -126), (100, 121)])
def test_scales_that_stay_and_scales_that_grow(new, scales):
    run(20, "bf16", "f32", 1, 3, 64, 64, 32, [45, 63, 70, 41], [min(new, 41)] * 4, 64, scales=scales)


@pytest.mark.parametrize("new", [1, 20])
def test_values_at_the_ends_of_the_range(new):
    """Zeros, the smallest and the largest numbers, infinities and NaN: of a token, of a head, of a whole block."""
    lens = [new + 3, new + 16, new]
    for k, (low, high) in enumerate([(0.0, 0.0), (1e-45, 1e-40), (1e-38, 3e-38), (1e37, 3.4028234e38), (126.9, 127.1), (np.inf, np.inf), (-np.inf, 1.0),
                                     (np.nan, np.nan), (1.0, np.nan)]):
        r = np.random.default_rng(100 + k)
        x = {}
        for n, h in (("k", 2), ("v", 2), ("q", 1)):
            v = r.standard_normal((3 * new, h, 64)).astype(np.float32)
            at = r.random(v.shape) < 0.3 if k % 2 else np.ones(v.shape, dtype=bool)
            pick = np.where(r.random(v.shape) < 0.5, np.float32(low), np.float32(high))
            x[n] = torch.from_numpy(np.where(at, pick, v).astype(np.float32))
        x["q"] = x["q"].nan_to_num(0.0, 1.0, -1.0).clamp(-1e30, 1e30)
        for rot in (0, 64):
            if rot:  # turned: every number must stay one, so that NaN and infinities come from the rows alone
                x["k"] = x["k"].clamp(-1e37, 1e37)
            run(21 + k, "bf16", "f32", 1, 2, 64, 32, 16, lens, [new] * 3, rot, x=x)


def test_numbers_half_way_between_two():
    """Ties go to the even one, of new values and of numbers that go into larger steps."""
    p = paged_i8(40, 1, 64, 16, 16, [9], [1])
    p["ks"][:] = p["vs"][:] = 1.0
    for old in (p["k"], p["v"]):
        old[:] = np.arange(-32, 32, dtype=np.int8)  # odd ones are half way when the steps double
    x = torch.arange(-32, 32, dtype=torch.float32).reshape(1, 1, 64) + 0.5
    x[0, 0, 0] = 200.0  # steps of 2: 1.5 is 0.75 steps, 3 half way between ..
    x[0, 0, 1:32] = torch.arange(-15, 16, dtype=torch.float32) * 2 + 1.0
    cache, t = device_cache_i8(p)
    xd = x.cuda()
    dc.kv_append(cache, device_batch(p), dc.KVRows(dc.TYPE_F32, 0, xd, xd), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    check(p, {"k": x, "v": x}, t, None, np.zeros((9, 0), np.float32), np.zeros((9, 0), np.float32), False)
    page = int(p["batch"]["pages"][0, 0])
    assert t[2][page, 0, 0] == 2.0
    assert t[0][page, 0, 0].tolist() == [int(np.rint(n / 2)) for n in range(-32, 32)]
    assert t[0][page, 0, 8, 1:32].tolist() == [int(np.rint(n + 0.5)) for n in range(-15, 16)]


@pytest.mark.parametrize("block", [16, 64])
def test_scales_do_not_depend_on_how_tokens_are_divided(block):
    print(f"case append i8 divided block={block}", flush=True)
    n, kv, d, page = 150, 2, 64, 64
    whole = paged_i8(41, kv, d, page, block, [n], [n])
    x = rows_of(whole, "f32", 1)
    st = torch.cuda.current_stream().cuda_stream
    kd, vd = x["k"].cuda(), x["v"].cuda()
    results = []
    for pieces in ([n], [1] * n, [7, 60, 1, 2, 80]):
        cache, t = device_cache_i8(whole)
        for s in t[2:]:
            s.fill_(float("nan"))
        at = 0
        for new in pieces:
            part = dict(whole, batch=dict(whole["batch"], lens=np.array([at + new], dtype=np.int32), starts=np.array([0, new], dtype=np.int32)), news=[new])
            dc.kv_append(cache, device_batch(part), dc.KVRows(dc.TYPE_F32, 0, kd[at:at + new], vd[at:at + new]), st)
            at += new
        torch.cuda.synchronize()
        results.append([a.cpu().numpy() for a in t])
    pages = whole["batch"]["pages"][0]
    for other in results[1:]:
        for i in (2, 3):
            s0, s1 = results[0][i][pages], other[i][pages]
            n_blocks = -(-n // block)
            flat = lambda s: s.transpose(0, 2, 1).reshape(-1, kv)[:n_blocks]  # noqa: E731
            assert np.array_equal(flat(s0), flat(s1))
        # a number is rounded once and then again to each larger step: one step in all at most
        for i in (0, 1):
            for j in range(n):
                a, b = (r[i][pages[j // page], :, j % page].astype(int) for r in (results[0], other))
                assert np.abs(a - b).max() <= 1


def test_another_stream():
    run(42, "bf16", "bf16", 4, 2, 128, 16, 16, [300, 20], [300, 4], 128, stream=torch.cuda.Stream())


@pytest.mark.parametrize("x_type", ["f32", "bf16"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("d,news", [(64, [3, 1]), (128, [100, 5]), (256, [2, 2])])
def test_rows_and_tables_at_odd_multiples_of_16_bytes(x_type, neighbours, d, news):
    print(f"case append i8 at 16 bytes {x_type} neighbours={neighbours} d={d} news={news}", flush=True)
    heads, kv, lens = 4, 2, [n + 7 for n in news]
    p = paged_i8(43, kv, d, 16, 16, lens, news)
    x = rows_of(p, x_type, heads)
    cos, sin = angles(max(lens), d // 2)
    skip = 16 // x["k"].element_size()
    kd, vd, qd = (_rows_at(torch, x[n].cuda(), skip) for n in ("k", "v", "q"))
    cd, sd = _rows_at(torch, torch.from_numpy(cos).cuda(), 4), _rows_at(torch, torch.from_numpy(sin).cuda(), 4)
    out = _rows_at(torch, torch.zeros((sum(news), heads, d), dtype=torch.bfloat16, device="cuda"), 8)
    pools = [torch.zeros(p[n].size + 64, dtype=torch.int8, device="cuda") for n in ("k", "v")]
    k, v = (w[-w.data_ptr() % 32 + 16:][:p["k"].size].view(p["k"].shape) for w in pools)
    k.copy_(torch.from_numpy(p["k"])), v.copy_(torch.from_numpy(p["v"]))
    wide = [torch.from_numpy(np.concatenate([[1.0], p[n].ravel()]).astype(np.float32)).cuda() for n in ("ks", "vs")]
    ks, vs = (w[1:].view(p["ks"].shape) for w in wide)  # at 4 bytes
    cache = dc.KVCache(k, v, p["n_pages"], kv, d, 16, dc.TYPE_I8, rows_type=dc.TYPE_BF16, scale_tokens=16, k_scale_dev=ks, v_scale_dev=vs)
    dc.kv_append(cache, device_batch(p), dc.KVRows(KIND[x_type], heads, kd, vd, qd, out, rot_dim=d, pairing=int(neighbours), cos_dev=cd, sin_dev=sd,
                                                   n_positions=max(lens)), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    check(p, x, (k, v, ks, vs), out, cos, sin, neighbours)


def test_queries_turned_in_place():
    p = paged_i8(44, 2, 128, 16, 16, [9, 30], [4, 6])
    x = torch.from_numpy(p["rng"].standard_normal((10, 8, 128)).astype(np.float32)).to(torch.bfloat16)
    cos, sin = angles(30, 64)
    for neighbours in (False, True):
        cache, t = device_cache_i8(p)
        rows = x.cuda()
        q, kk, vv = rows[:, :4], rows[:, 4:6], rows[:, 6:]
        cd, sd = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
        dc.kv_append(cache, device_batch(p), dc.KVRows(dc.TYPE_BF16, 4, kk, vv, q, q, rot_dim=128, pairing=int(neighbours), cos_dev=cd, sin_dev=sd,
                                                       n_positions=30), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        check(p, {"k": x[:, 4:6], "v": x[:, 6:], "q": x[:, :4]}, t, q, cos, sin, neighbours)
        assert torch.equal(rows[:, 4:].cpu(), x[:, 4:])


def test_pages_beyond_four_gib():
    d, page, kv, block = 128, 256, 8, 64
    n_pages = (5 << 30) // (page * kv * d)
    print(f"case append i8 pool of {n_pages} pages", flush=True)
    p = paged_i8(45, kv, d, page, block, [300, 270], [1, 120])
    x = rows_of(p, "bf16", 1)
    far = n_pages - p["n_pages"]
    pools = [torch.zeros((n_pages, kv, page, d), dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.full((n_pages, kv, page // block), float("nan"), device="cuda") for _ in range(2)]
    for big, small in zip(pools + scales, ("k", "v", "ks", "vs")):
        big[far:] = torch.from_numpy(p[small]).cuda()
    there = dict(p, batch=dict(p["batch"], pages=np.where(p["batch"]["pages"] >= 0, p["batch"]["pages"] + far, -1).astype(np.int32)))
    cache = dc.KVCache(pools[0], pools[1], n_pages, kv, d, page, dc.TYPE_I8, scale_tokens=block, k_scale_dev=scales[0], v_scale_dev=scales[1])
    kd, vd = x["k"].cuda(), x["v"].cuda()
    dc.kv_append(cache, device_batch(there), dc.KVRows(dc.TYPE_BF16, 0, kd, vd), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    check(p, x, [t[far:] for t in pools + scales], None, np.zeros((300, 0), np.float32), np.zeros((300, 0), np.float32), False)
    assert not any(bool(t[:far].any()) for t in pools) and all(bool(t[:far].isnan().all()) for t in scales)


def test_device_arrays_that_do_not_fit_are_survived():
    """Rows, lengths and pages outside what the call was told of: the other sequences' tokens are right, nothing outside is written."""
    p = paged_i8(46, 2, 64, 16, 16, [100, 60, 30], [8, 7, 9])
    x = rows_of(p, "f32", 1)
    kd, vd = x["k"].cuda(), x["v"].cuda()
    none = np.zeros((100, 0), np.float32)
    for lens in ([100, 60, 2 ** 31 - 1], [100, 60, -5], [100, 60, 31 + 16 * 7]):
        other = dict(p, batch=dict(p["batch"], lens=np.array(lens, dtype=np.int32)))
        cache, t = device_cache_i8(other)
        dc.kv_append(cache, device_batch(other, max_len=100), dc.KVRows(dc.TYPE_F32, 0, kd, vd), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        check(other, x, t, None, none, none, False)
    for starts in ([0, 8, 15, 2 ** 31 - 1], [0, 8, 15, -7], [0, 8, 15, 15], [-3, 8, 15, 24], [24, 24, 24, 24], [30, 20, 10, 0]):
        other = dict(p, batch=dict(p["batch"], starts=np.array(starts, dtype=np.int32)))
        arrays, skip = (p["k"], p["v"], p["ks"], p["vs"]), (16, 16, 1, 1)
        wide = [torch.full((a.size + 2 * s,), 99, dtype=torch.int8 if s == 16 else torch.float32, device="cuda") for a, s in zip(arrays, skip)]
        inner = [w[s:-s].view(a.shape) for w, s, a in zip(wide, skip, arrays)]
        cache = dc.KVCache(inner[0], inner[1], p["n_pages"], 2, 64, 16, dc.TYPE_I8, scale_tokens=16, k_scale_dev=inner[2], v_scale_dev=inner[3])
        dev = {n: torch.from_numpy(np.ascontiguousarray(other["batch"][n])).cuda() for n in ("lens", "starts", "pages")}
        batch = dc.KVBatch(3, 24, 24, 100, dev["lens"], dev["pages"], p["batch"]["pages"].shape[1], row_start_dev=dev["starts"])
        dc.kv_append(cache, batch, dc.KVRows(dc.TYPE_F32, 0, kd, vd), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all(bool((w[:s] == 99).all() and (w[-s:] == 99).all()) for w, s in zip(wide, skip))


@pytest.mark.parametrize("news", [[4, 30], [1, 1]])
def test_replays_of_a_recorded_call(news):
    p = paged_i8(47, 2, 64, 16, 16, [44, 39], news)
    x = rows_of(p, "f32", 4)
    cos, sin = angles(44, 32)
    cache, t = device_cache_i8(p)
    start = [a.clone() for a in t]
    batch = device_batch(p)
    rows = sum(news)
    out = torch.zeros((rows, 4, 64), dtype=torch.bfloat16, device="cuda")
    dev = {n: a.cuda() for n, a in x.items()}
    cd, sd = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    r = dc.KVRows(dc.TYPE_F32, 4, dev["k"], dev["v"], dev["q"], out, rot_dim=64, cos_dev=cd, sin_dev=sd, n_positions=44)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        dc.kv_append(cache, batch, r, side.cuda_stream)
    for _ in range(4):
        for a, s in zip(t, start):
            a.copy_(s)
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        check(p, x, t, out, cos, sin, False)
