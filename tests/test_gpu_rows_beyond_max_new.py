"""A sequence with more rows than the batch's max_new: its first max_new rows are served, the others are left alone by both calls."""
import numpy as np
import pytest

import oracle.attention as oa
import paper_2502_15443_amd as dc
from tests.attention_cases import KIND, SMALLEST, UNIT, check_attend, device_batch, device_cache, f64, paged, torch_type
from tests.test_gpu_attention import SENTINEL, attend, queries
from tests.test_gpu_kv_append import angles

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def beyond(news, max_new):
    """For every row whether it is one that is left alone."""
    return np.concatenate([np.arange(n) >= max_new for n in news])


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,news,max_new", [(4, 2, 64, [5, 2, 4], 3), (6, 1, 128, [1, 7, 1], 1), (4, 4, 256, [4, 4], 4),
                                                           (4, 2, 64, [400, 150, 3], 149), (24, 8, 128, [300, 260], 200)])  # few rows, many
def test_append(heads, kv_heads, d, news, max_new, neighbours, in_place):
    print(f"case append beyond max_new heads={heads}/{kv_heads} d={d} news={news} max_new={max_new}", flush=True)
    type, lens = "bf16", [n + 20 for n in news]
    p = paged(71, type, kv_heads, d, 32, lens, news, fill=SENTINEL)
    rows = sum(news)
    x = torch.from_numpy(p["rng"].standard_normal((rows, heads + 2 * kv_heads, d)).astype(np.float32)).to(torch_type(type))
    cos, sin = angles(max(lens), d // 2)
    cache, k, v = device_cache(p)
    batch = device_batch(dict(p, news=[max_new]))
    assert batch.max_new == max_new
    xd = x.cuda()
    q, kd, vd = xd.split([heads, kv_heads, kv_heads], dim=1)
    out = q if in_place else torch.full((rows, heads, d), SENTINEL, dtype=x.dtype, device="cuda")
    before = f64(out)
    dc.kv_append(cache, batch, dc.KVRows(KIND[type], heads, kd, vd, q, out, rot_dim=d, pairing=int(neighbours), cos_dev=torch.from_numpy(cos).cuda(),
                                         sin_dev=torch.from_numpy(sin).cuda(), n_positions=max(lens)), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    left = beyond(news, max_new)
    assert left.any() == (max(news) > max_new)
    # rows that are left alone: the oracle is given no cosines for them
    positions = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, news)])
    xk, xv, xq = (f64(t) for t in (x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], x[:, :heads]))
    want_k, want_v, want_q = oa.append(f64(p["k"]), f64(p["v"]), p["batch"], xk, xv, xq, cos.astype(np.float64), sin.astype(np.float64), neighbours,
                                       np.where(left, -1, positions))
    def near(got, want):  # written once: two products and a sum of values of at most `most` in fp32, then rounded
        tol = UNIT[type] * np.abs(want) * 1.001 + 4 * 2.0 ** -24 * 2 * float(x.abs().max()) + SMALLEST[type]
        return (np.abs(got - want) <= tol).all()
    got = f64(out)
    assert np.array_equal(got[left], before[left]) and near(got[~left], want_q[~left])
    assert np.array_equal(f64(v), want_v) and near(f64(k), want_k)
    untouched = want_k == f64(p["k"])
    assert np.array_equal(f64(k)[untouched], f64(p["k"])[untouched])


@pytest.mark.parametrize("heads,kv_heads,d,news,max_new,prefix", [
    (4, 2, 64, [5, 2, 4], 3, 0), (8, 2, 128, [8, 1, 5], 7, 0),                      # few rows of a sequence
    (4, 1, 64, [60, 20], 40, 0), (2, 1, 128, [200, 129, 5], 128, 0), (4, 2, 256, [40, 70], 35, 0),  # many
    (4, 2, 64, [3, 2], 1, 75),                                                      # a prefix and few rows
    (9, 1, 128, [2] * 20, 1, 130), (9, 1, 64, [3] * 20, 2, 130),                    # few rows of a sequence, many of the batch
    (4, 2, 64, [70, 64], 50, 130), (1, 1, 256, [150, 140], 129, 40),                # the prefix along with the own pages
    (5, 1, 64, [9] * 12, 8, 7003),                                                  # the prefix apart, many rows of a sequence
])
def test_attention(heads, kv_heads, d, news, max_new, prefix):
    print(f"case attention beyond max_new heads={heads}/{kv_heads} d={d} news={news} max_new={max_new} prefix={prefix}", flush=True)
    p = paged(72, "bf16", kv_heads, d, 32, [prefix + n + 30 for n in news], news, prefix)
    q = queries(p, heads, "bf16")
    got, got_lse = attend(dict(p, news=[max_new]), heads, q, d ** -0.5)
    left = beyond(news, max_new)
    assert left.any()
    assert (got[left] == SENTINEL).all() and (got_lse[left] == SENTINEL).all()
    out, lse, size = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q), np.float64(np.float32(d ** -0.5)))
    kept = {k: v[~left] for k, v in size.items()}
    check_attend("bf16", d, got[~left], got_lse[~left], out[~left], lse[~left], kept)
