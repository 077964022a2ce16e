"""dc_kv_append and each kernel of dc_attention_paged on pages beyond 2^32 bytes and 2^31 elements of the pools, every result compared; and a
common prefix some of whose pages are not there, or inside which sequences end."""
import numpy as np
import pytest

import oracle.attention as oa
import paper_2502_15443_amd as dc
from tests.attention_cases import KIND, UNIT, check_attend, f64, paged
from tests.test_gpu_attention import attend, queries
from tests.test_gpu_kv_append import angles

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pools():
    """Keys and values of 5 GiB each: [pages, 4, 256, 128] in bf16."""
    shape = ((5 << 30) // (4 * 256 * 128 * 2), 4, 256, 128)
    k = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    yield k, v


def moved(p, pools):
    """The problem with its pages at the end of the pools; near pages are NaN, so that what is read there by mistake is seen."""
    k, v = pools
    far = k.shape[0] - p["n_pages"]
    assert far * k[0].numel() > 2 ** 31
    for pool, x in ((k, p["k"]), (v, p["v"])):
        pool[:far].fill_(float("nan"))
        pool[far:] = x.cuda()
    b = p["batch"]
    table = torch.from_numpy(np.where(b["pages"] >= 0, b["pages"] + far, -1).astype(np.int32)).cuda()
    prefix = torch.from_numpy((b["prefix_pages"] + far).astype(np.int32)).cuda()
    lens, starts = torch.from_numpy(b["lens"]).cuda(), torch.from_numpy(b["starts"]).cuda()
    cache = dc.KVCache(k, v, k.shape[0], 4, 128, 256, KIND["bf16"])
    batch = dc.KVBatch(len(b["lens"]), int(b["starts"][-1]), max(p["news"]), int(b["lens"].max()), lens, table, table.shape[1], row_start_dev=starts,
                       prefix_len=b["prefix_len"], prefix_pages_dev=prefix if b["prefix_len"] else None)
    return cache, batch, far


@pytest.mark.parametrize("heads,news,prefix", [(4, [1], 0), (4, [30, 2], 0), (4, [130, 200], 0), (40, [5, 9], 0),  # few rows and many
                                               (4, [1, 2], 300), (40, [3, 3, 3], 300), (8, [60, 40], 300)])       # with a prefix, each way
def test_attention(pools, heads, news, prefix):
    print(f"case far pages attention heads={heads} news={news} prefix={prefix}", flush=True)
    p = paged(101, "bf16", 4, 128, 256, [prefix + n + 260 for n in news], news, prefix)
    cache, batch, _ = moved(p, pools)
    q = queries(p, heads, "bf16")
    qd = q.cuda()
    out, lse = torch.empty_like(qd), torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    a = dc.Attention(heads, qd, out, lse, 0.1)
    n = dc.attention_paged_workspace(cache, batch, a)
    dc.attention_paged(cache, batch, a, torch.empty(n + 16, dtype=torch.uint8, device="cuda"), n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    want = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q), np.float64(np.float32(0.1)))
    check_attend("bf16", 128, f64(out), f64(lse), *want)


@pytest.mark.parametrize("news", [[3, 1], [600, 40]])  # few rows, many
def test_append(pools, news):
    print(f"case far pages append news={news}", flush=True)
    lens = [n + 300 for n in news]
    p = paged(102, "bf16", 4, 128, 256, lens, news, fill=7.75)
    cache, batch, far = moved(p, pools)
    rows = sum(news)
    x = torch.from_numpy(p["rng"].standard_normal((rows, 12, 128)).astype(np.float32)).to(torch.bfloat16)
    q, kk, vv = x.cuda().split([4, 4, 4], dim=1)
    cos, sin = angles(max(lens), 64)
    out = torch.empty((rows, 4, 128), dtype=torch.bfloat16, device="cuda")
    dc.kv_append(cache, batch, dc.KVRows(KIND["bf16"], 4, kk, vv, q, out, rot_dim=128, cos_dev=torch.from_numpy(cos).cuda(), sin_dev=torch.from_numpy(sin).cuda(),
                                         n_positions=max(lens)), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    want_k, want_v, want_q = oa.append(f64(p["k"]), f64(p["v"]), p["batch"], f64(x[:, 4:8]), f64(x[:, 8:]), f64(x[:, :4]), cos.astype(np.float64),
                                       sin.astype(np.float64), False)
    for got, want in ((pools[0][far:], want_k), (pools[1][far:], want_v), (out, want_q)):
        assert (np.abs(f64(got) - want) <= UNIT["bf16"] * np.abs(want) * 1.001 + 2.0 ** -21 * 5).all()
    for pool in pools:  # nothing near the beginning was written
        assert torch.isnan(pool[:far]).all()


@pytest.mark.parametrize("heads,kv_heads,news", [(4, 2, [1, 1, 3]), (9, 1, [2] * 20), (4, 1, [60, 40])])  # few rows; many of the batch; many of each
@pytest.mark.parametrize("gone", [[0], [1, 3], [4], [0, 1, 2, 3, 4]])
def test_prefix_pages_that_are_not_there(heads, kv_heads, news, gone):
    print(f"case absent prefix pages heads={heads}/{kv_heads} news={news} gone={gone}", flush=True)
    prefix = 70
    p = paged(103, "bf16", kv_heads, 64, 16, [prefix + n + 5 for n in news], news, prefix)
    for i in gone:
        p["batch"]["prefix_pages"][i] = [-1, p["n_pages"], 2 ** 31 - 1][i % 3]
    q = queries(p, heads, "bf16")
    got, got_lse = attend(p, heads, q, 0.125)
    want = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q), 0.125)
    check_attend("bf16", 64, got, got_lse, *want)


@pytest.mark.parametrize("heads,kv_heads,d,news", [(4, 2, 64, [1, 3, 1]), (9, 1, 128, [2, 1] * 10), (4, 1, 64, [60, 40, 33]), (2, 1, 256, [70, 64, 5])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 2)])
def test_sequences_that_end_inside_the_prefix(heads, kv_heads, d, news, window, sinks):
    print(f"case ends inside the prefix heads={heads}/{kv_heads} d={d} news={news} window={window}", flush=True)
    prefix = 150
    lens = [[140, 150, 75, 170][i % 4] for i in range(len(news))]
    p = paged(104, "bf16", kv_heads, d, 16, lens, news, prefix)
    q = queries(p, heads, "bf16")
    got, got_lse = attend(p, heads, q, 0.125, window, sinks)
    want = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q), 0.125, window, sinks)
    check_attend("bf16", d, got, got_lse, *want)
