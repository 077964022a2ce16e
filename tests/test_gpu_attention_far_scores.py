"""dc_attention_paged where the first keys' scores lie far below those of later ones: the later ones, which alone carry weight, keep their
precision whatever came before them."""
import numpy as np
import pytest

import oracle.attention as oa
from tests.attention_cases import check_attend, f64, paged
from tests.test_gpu_attention import attend, queries

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("news,heads", [(1, 1), (9, 3), (140, 1), (60, 4)])  # of each of the kernels
@pytest.mark.parametrize("prefix", [0, 64])
@pytest.mark.parametrize("far", [2.0 ** 7, 2.0 ** 15])  # scores of -2^14 or -2^30 before the scale
@pytest.mark.parametrize("max_len", [None, 1])  # runs of keys cut in parts; in one part, with the far scores at its beginning
def test_ordinary_scores_behind_far_lower_ones(type, d, news, heads, prefix, far, max_len):
    print(f"case far scores {type} d={d} news={news} heads={heads} prefix={prefix} far={far} max_len={max_len}", flush=True)
    page = 64
    lens, rows = [500, 410], [news, news]
    p = paged(61, type, 1, d, page, lens, rows, prefix)
    q = queries(p, heads, type)
    q[:, :, 0] = far
    # tokens of the first page: a far lower score; of the others: ordinary ones, that rise along the keys
    for b, n in enumerate(lens):
        for j in range(n):
            pg, at = oa.place_of(p["batch"], b, j, page, p["n_pages"])
            p["k"][pg, :, at, 0] = -far if j < page else 0.0
            if prefix == 0 or j >= prefix:
                p["k"][pg, :, at, 1:] *= 1.0 + j / 200
    got, got_lse = attend(p, heads, q, d ** -0.5, uniform=news == 1, max_len=max_len)
    # in 64 bits those first tokens have no weight at all: the result is that without their page, and so are the sizes that its error goes by
    scale = np.float64(np.float32(d ** -0.5))
    without = dict(p["batch"], pages=p["batch"]["pages"].copy(), prefix_pages=p["batch"]["prefix_pages"].copy())
    if prefix:
        without["prefix_pages"][0] = -1
    else:
        without["pages"][:, 0] = -1
    out, lse, size = oa.attend(f64(p["k"]), f64(p["v"]), without, f64(q), scale)
    whole, whole_lse, _ = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q), scale)
    assert np.allclose(out, whole, rtol=1e-12, atol=0) and np.allclose(lse, whole_lse, rtol=1e-12, atol=0)
    check_attend(type, d, got, got_lse, out, lse, size)
