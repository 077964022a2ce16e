"""Scales of dc_attention_paged: the kernels multiply scores by scale * log2(e), which has to be a number of fp32."""
import pytest

import paper_2502_15443_amd as dc

ADDR = 1 << 20


@pytest.mark.parametrize("scale,good", [(2.0 ** 127, True), (-2.0 ** 127, True), (2.0 ** 127 * 1.01, False), (3.4e38, False), (-3.4e38, False), (1e-45, True)])
def test_scales_that_are_too_large_are_refused(scale, good):
    cache = dc.KVCache(ADDR, ADDR, 10, 2, 128, 16, dc.TYPE_BF16)
    batch = dc.KVBatch(1, 1, 1, 100, ADDR, ADDR, 7)
    s = (512, 128)
    a = dc.Attention(4, ADDR, 2 * ADDR, None, scale, q_strides=s, out_strides=s)
    if good:
        dc.attention_paged_workspace(cache, batch, a)
        return
    for call in (lambda: dc.attention_paged_workspace(cache, batch, a), lambda: dc.attention_paged(cache, batch, a, ADDR, 1 << 40)):
        with pytest.raises(dc.DCError) as e:
            call()
        assert e.value.code == -1


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("news", [1, 140])  # of each kernel
@pytest.mark.parametrize("scale", [2.0 ** 127, -2.0 ** 127, 1e-45])
def test_scales_at_the_ends(type, news, scale):
    """One key agrees with the query in one value, the others have nothing in common with it: all of the weight, or an equal share."""
    torch = pytest.importorskip("torch")
    import numpy as np

    import oracle.attention as oa
    from tests.attention_cases import UNIT, f64, paged
    from tests.test_gpu_attention import attend

    print(f"case scale {scale} {type} news={news}", flush=True)
    length, d = 200, 64
    p = paged(95, type, 1, d, 16, [length], [news])
    q = torch.zeros((news, 1, d), dtype=p["k"].dtype)
    q[:, :, 0] = 2.0 ** -10
    for j in range(length):
        page, at = oa.place_of(p["batch"], 0, j, 16, p["n_pages"])
        p["k"][page, :, at] = 0
        p["k"][page, :, at, 0] = (1 if scale > 0 else -1) * 2.0 ** -10 if j == 30 else 0.0
    got, got_lse = attend(p, 1, q, scale, uniform=news == 1)
    values = np.stack([f64(p["v"])[pg, 0, at] for pg, at in (oa.place_of(p["batch"], 0, j, 16, p["n_pages"]) for j in range(length))])
    for row in range(news):
        n = length - news + row + 1  # keys that the row sees
        if abs(scale) > 1 and n > 30:
            want, lse = values[30], 2.0 ** 107
        else:
            want, lse = values[:n].mean(0), np.log(n)
        # weights 1 and one rounding; a mean of n values in fp32
        assert (np.abs(got[row, 0] - want) <= UNIT[type] * np.abs(want) + 2 * n * 2.0 ** -24 * np.abs(values[:n]).max()).all()
        assert abs(got_lse[row, 0] - lse) <= 8 * 2.0 ** -24 * abs(lse) + 2.0 ** -20


@pytest.mark.gpu
@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("news,heads", [(5, 2), (140, 1)])  # of each kernel
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_queries_that_are_no_numbers_with_a_scale_of_zero(type, d, news, heads, value):
    """0 times a score that is no number is none; rows of numbers take the mean of their values."""
    torch = pytest.importorskip("torch")
    import numpy as np

    import oracle.attention as oa
    from tests.attention_cases import check_attend, f64, paged
    from tests.test_gpu_attention import attend, queries

    print(f"case scale 0 {type} d={d} news={news} {value}", flush=True)
    p = paged(96, type, 1, d, 16, [200], [news])
    q = queries(p, heads, type)
    out, lse, size = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q), 0.0)
    q[2, 0, 5] = value
    got, got_lse = attend(p, heads, q, 0.0)
    assert np.isnan(got[2, 0]).all() and np.isnan(got_lse[2, 0])
    got[2, 0], got_lse[2, 0] = out[2, 0], lse[2, 0]
    check_attend(type, d, got, got_lse, out, lse, size)
