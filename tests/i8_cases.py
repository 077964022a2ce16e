"""Problems for the tests of the cache held in 8 bits, and the tolerances of its attention's results."""
from __future__ import annotations

import numpy as np

import oracle.attention as oa
import oracle.cache_i8 as oc8
import paper_2502_15443_amd as dc
from tests.attention_cases import KIND, SMALLEST, UNIT

ODD = [np.nan, np.inf, -1.0, 0.0, 3e38]


def paged_i8(seed, kv_heads, head_dim, page, block, lens, news, prefix=0, absent=(), spare=3, rows_type="bf16", scales=(-6, -4)):
    """A cache of 8 bits and a batch.  Pages are in random order; numbers of no token are any bytes, scales of blocks without tokens no
    sound ones.  Returns a dict; scales are powers of two with exponents in `scales`."""
    r = np.random.default_rng(seed)
    private = [max(0, n - prefix) for n in lens]
    stride = max(1, max(-(-p // page) for p in private))
    prefix_pages = -(-prefix // page)
    n_pages = prefix_pages + len(lens) * stride + spare
    order = r.permutation(n_pages)
    table = np.full((len(lens), stride), -1, dtype=np.int32)
    for b, p in enumerate(private):
        for i in range(-(-p // page)):
            table[b, i] = order[prefix_pages + b * stride + i]
    for b, i in absent:
        table[b, i] = [-1, n_pages, -2 ** 31, 2 ** 31 - 1][(b + i) % 4]
    batch = {"lens": np.array(lens, dtype=np.int32), "starts": np.concatenate([[0], np.cumsum(news)]).astype(np.int32),
             "pages": table, "prefix_len": prefix, "prefix_pages": order[:prefix_pages].astype(np.int32)}
    held = np.zeros((n_pages, page // block), dtype=bool)  # blocks with a token
    tokens = np.zeros((n_pages, page), dtype=bool)
    for b, n in enumerate(lens):
        for j in range(n):
            w = oa.place_of(batch, b, j, page, n_pages)
            if w is not None:
                held[w[0], w[1] // block] = tokens[w] = True
    pools, pool_scales = [], []
    for _ in range(2):
        x = r.integers(-128, 128, (n_pages, kv_heads, page, head_dim)).astype(np.int8)
        values = np.clip(np.rint(r.standard_normal(x.shape) * 32), -127, 127).astype(np.int8)
        pools.append(np.where(tokens[:, None, :, None], values, x))
        s = (2.0 ** r.integers(scales[0], scales[1] + 1, (n_pages, kv_heads, page // block))).astype(np.float32)
        odd = np.array(ODD, dtype=np.float32)[r.integers(0, len(ODD), s.shape)]
        pool_scales.append(np.where(held[:, None, :], s, odd))
    return {"type": rows_type, "page": page, "block": block, "k": pools[0], "v": pools[1], "ks": pool_scales[0], "vs": pool_scales[1], "batch": batch,
            "n_pages": n_pages, "kv_heads": kv_heads, "head_dim": head_dim, "news": list(news), "rng": r}


def device_cache_i8(p):
    """(cache, pools and scales on the GPU)"""
    import torch

    t = [torch.from_numpy(p[n].copy()).cuda() for n in ("k", "v", "ks", "vs")]
    return dc.KVCache(t[0], t[1], p["n_pages"], p["kv_heads"], p["head_dim"], p["page"], dc.TYPE_I8, rows_type=KIND[p["type"]],
                      scale_tokens=p["block"], k_scale_dev=t[2], v_scale_dev=t[3]), t


def pool_values(p):
    """Keys and values in fp64."""
    return oc8.values(p["k"], p["ks"]), oc8.values(p["v"], p["vs"])


def check_attend_i8(type, d, got, got_lse, out, lse, size, most_scale):
    """Keys and queries enter their product as they are.  With e = 2^-24: a score is off by at most (d + 12) e of its largest sum of |q k|
    (d additions, the scale of the block and of the call, the reference), and an error x of a score changes its weight by the factor 1 + x;
    sums over n keys add at most n e, exp, log and the joining of parts a few e.  A weight times its value's scale is rounded to f16, relative
    2^-11.  Below f16's normal range that is 2^-25 at most of a number that stands for weight 2^-7 at the largest value scale, rounded up to a power of two
    (`most_scale` at most), while the weights' sum is at least 1 and the numbers are at most 128: 2^-32 * most_scale * 128 a key.  The result is rounded to
    the rows' type once."""
    e = 2.0 ** -24
    small = e * (2 * (d + 12) * size["s"] + 2 * size["n"][:, None] + 64 + 4 * np.abs(np.where(np.isfinite(lse), lse, 0)))
    tol = size["v"] * (1.01 * (UNIT["f16"] + UNIT[type]) + 2 * small[:, :, None]) + 2.0 ** -25 * most_scale * size["n"][:, None, None] + SMALLEST[type]
    served = ~np.isnan(lse)
    nothing = np.isneginf(lse) & served
    assert (got[nothing] == 0).all() and np.isneginf(got_lse[nothing]).all()
    some = served & ~nothing
    assert np.isfinite(got[some]).all() and np.isfinite(got_lse[some]).all()
    off, off_lse = np.abs(got - out)[some], np.abs(got_lse[some] - lse[some])
    assert (off <= tol[some]).all(), ("out", float((off / tol[some]).max()), float(off.max()))
    assert (off_lse <= 2 * small[some]).all(), ("lse", float((off_lse / (2 * small[some])).max()))
