"""dc_kv_append into blocks of a cache of 8 bits whose scales are no powers of two (a program may have written them): new values become the whole numbers nearest
to x / s, and earlier numbers the nearest to what they stood for, also where x / s lies next to the middle between two whole numbers."""
from fractions import Fraction

import numpy as np
import pytest

import oracle.attention as oa
import oracle.cache_i8 as oc8


def near_the_middle(r, scale, shape):
    """fp32 values that are a scale times half an odd number, up to 126.5, or next to it."""
    x = ((r.integers(-126, 126, shape) + 0.5) * np.float64(scale)).astype(np.float32)
    step = r.integers(-1, 2, shape)
    return np.where(step, np.nextafter(x, np.where(step > 0, np.float32(np.inf), np.float32(-np.inf))), x).astype(np.float32)


def odd_scale(r, low=-8, high=-4):
    """Half of them such that a whole number up to 127 times the scale is next to the middle between two."""
    if r.random() < 0.5:
        q = int(r.integers(3, 128))
        return np.float32((2 * int(r.integers(q // 4, q // 2)) + 1) / (2 * q) * 2.0 ** int(r.integers(low, high + 1)))
    return np.float32(r.uniform(0.5, 1.0) * 2.0 ** int(r.integers(low, high + 1)))


def exact(x, s):
    q = Fraction(float(x)) / Fraction(float(s))
    return round(q)  # ties to even


def test_the_oracle_is_exact():
    r = np.random.default_rng(1)
    for _ in range(300):
        s = odd_scale(r, -120, 120)
        x = near_the_middle(r, s, 50)
        assert oc8.whole(x, s).tolist() == [exact(v, s) for v in x]


def test_the_oracle_holds_earlier_numbers_exactly():
    r = np.random.default_rng(2)
    for _ in range(100):
        s = odd_scale(r)
        k = r.integers(-127, 128, (1, 1, 16, 64)).astype(np.int8)
        ks, x = np.full((1, 1, 1), s), np.full((1, 1, 64), s * 200, np.float32)
        b = {"lens": [9], "starts": [0, 1], "pages": np.array([[0]]), "prefix_len": 0, "prefix_pages": []}
        k2, _, ks2, _ = oc8.append(k, k, ks, ks, b, 16, x, x, None, None, False)
        grown = ks2[0, 0, 0]
        assert grown > s and np.log2(grown) % 1 == 0
        assert k2[0, 0, :8].ravel().tolist() == [round(int(q) * Fraction(float(s)) / Fraction(float(grown))) for q in k[0, 0, :8].ravel()]


def problem(seed, kv_heads, d, page, block, lens, news, grows, powers):
    """Blocks with earlier tokens have scales that are no powers of two; new values are next to the middle between two numbers, or make the scale grow."""
    from tests.i8_cases import paged_i8

    p = paged_i8(seed, kv_heads, d, page, block, lens, news)
    r = p["rng"]
    for n in ("ks", "vs"):
        p[n] = np.where(np.isfinite(p[n]) & (p[n] > 0) & (p[n] < 1), np.vectorize(lambda s: odd_scale(r, *powers))(p[n]), p[n]).astype(np.float32)
    x, most = {}, np.float32(2.0 ** (powers[1] + 1))
    for name, scales in (("k", "ks"), ("v", "vs")):
        x[name] = np.zeros((sum(news), kv_heads, d), np.float32)
        for b, length in enumerate(lens):
            for i in range(news[b]):
                w = oa.place_of(p["batch"], b, length - news[b] + i, page, p["n_pages"])
                for h in range(kv_heads):
                    row, scale = int(p["batch"]["starts"][b]) + i, min(oc8.sound(p[scales][w[0], h, w[1] // block]), most)
                    x[name][row, h] = near_the_middle(r, scale, d)
                    if grows:
                        x[name][row, h, int(r.integers(d))] = scale * np.float32(r.uniform(130, 500))
    return p, x


@pytest.mark.gpu
@pytest.mark.parametrize("grows", [False, True])
@pytest.mark.parametrize("d,page,block", [(64, 32, 16), (128, 16, 16), (64, 32, 32), (256, 32, 32), (128, 64, 64), (128, 256, 256), (256, 128, 128)])
@pytest.mark.parametrize("x_type,powers", [("f32", (-8, -4)), ("bf16", (-8, -4)), ("f32", (3, 6)), ("f32", (-126, -118)), ("bf16", (110, 117))])
def test_scales_that_are_no_powers_of_two(d, page, block, grows, x_type, powers):
    torch = pytest.importorskip("torch")
    import paper_2502_15443_amd as dc
    from tests.attention_cases import KIND, device_batch, torch_type
    from tests.i8_cases import device_cache_i8
    from tests.test_gpu_kv_append_i8 import check

    for seed, (lens, news) in enumerate([([block // 2 + 1, block - 1, block + 3], [1, 3, 2]), ([block + block // 2, 2 * block - 1, block // 2 + 9], [12, block - 2, 9]),
                                         ([3 * block + 5], [2 * block - 1])]):
        p, x = problem(seed + 1, 2, d, page, block, lens, news, grows, powers)
        x = {n: torch.from_numpy(v).to(torch_type(x_type)) for n, v in x.items()}
        print(f"case append i8 any scale {x_type} d={d} page={page} block={block} lens={lens} news={news} grows={grows} powers={powers}", flush=True)
        cache, t = device_cache_i8(p)
        kd, vd = x["k"].cuda(), x["v"].cuda()
        dc.kv_append(cache, device_batch(p), dc.KVRows(KIND[x_type], 0, kd, vd, None, None), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        check(p, x, t, None, None, None, False)
