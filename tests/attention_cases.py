"""Problems for the tests of the cache append and of the attention over a paged cache, and the tolerances of their results."""
from __future__ import annotations

import numpy as np

import oracle.attention as oa
import paper_2502_15443_amd as dc

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}  # relative error of one rounding: 8, 11 and 24 significant bits
SMALLEST = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}  # absolute error of one rounding below the normal range
KIND = {"bf16": dc.TYPE_BF16, "f16": dc.TYPE_F16, "f32": dc.TYPE_F32}


def torch_type(name):
    import torch

    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


def paged(seed, type, kv_heads, head_dim, page, lens, news, prefix=0, absent=(), spare=3, fill=float("nan")):
    """A cache and a batch: pages in random order, every value that belongs to no token is `fill`.  absent: (sequence, table
    entry) pairs that are not there.  Returns a dict; values are those of the type, as fp64."""
    import torch

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
    shape = (n_pages, kv_heads, page, head_dim)
    t = torch_type(type)
    pools = []
    for _ in range(2):
        x = torch.full(shape, fill, dtype=t)
        values = torch.from_numpy(r.standard_normal(shape).astype(np.float32)).to(t)
        for b, n in enumerate(lens):
            for j in range(n):
                w = oa.place_of(batch, b, j, page, n_pages)
                if w is not None:
                    x[w[0], :, w[1]] = values[w[0], :, w[1]]
        pools.append(x)
    return {"type": type, "page": page, "k": pools[0], "v": pools[1], "batch": batch, "n_pages": n_pages, "kv_heads": kv_heads,
            "head_dim": head_dim, "news": list(news), "rng": r}


def f64(x):
    import torch

    return x.to(torch.float64).cpu().numpy()


def rows_tensor(x, layout):
    """x [rows, heads, d] on the GPU in one of several layouts: dense, heads first, or a slice of wider rows."""
    import torch

    rows, heads, d = x.shape
    if layout == "heads first":
        y = torch.full((heads, rows, d), float("nan"), dtype=x.dtype, device="cuda").transpose(0, 1)
    elif layout == "slice":
        y = torch.full((rows, heads + 3, d + 8), float("nan"), dtype=x.dtype, device="cuda")[:, 1:1 + heads, 8:]
    else:
        y = torch.empty((rows, heads, d), dtype=x.dtype, device="cuda")
    y.copy_(x)
    return y


def device_batch(p, uniform=False, max_len=None):
    import torch

    b = p["batch"]
    dev = {k: torch.from_numpy(np.ascontiguousarray(b[k])).cuda() for k in ("lens", "starts", "pages", "prefix_pages")}
    rows = int(b["starts"][-1])
    return dc.KVBatch(len(b["lens"]), rows, max(1, max(p["news"])), max_len or max(1, int(b["lens"].max())), dev["lens"], dev["pages"],
                      b["pages"].shape[1], row_start_dev=None if uniform else dev["starts"], prefix_len=b["prefix_len"],
                      prefix_pages_dev=dev["prefix_pages"] if b["prefix_len"] else None)


def device_cache(p):
    k, v = p["k"].cuda(), p["v"].cuda()
    return dc.KVCache(k, v, p["n_pages"], p["kv_heads"], p["head_dim"], p["page"], KIND[p["type"]]), k, v


def attend_tolerance(type, d, out, lse, size):
    """(of out, of lse), element by element.  With u the unit of the type and e = 2^-24: every weight exp(s - reference) is rounded to
    the type once, relative u (absolute below its normal range; the weights' sum is at least 1), and the result is rounded once:
    2 u of the average over |v|.  A score is off by at most (d + 8) e of its largest sum of |q k| and rounding of the scale, and an
    error x of a score changes its weight by the factor 1 + x; sums over n keys add at most n e, exp, log and the joining of parts a few e."""
    u, e = UNIT[type], 2.0 ** -24
    small = e * (2 * (d + 8) * size["s"] + 2 * size["n"][:, None] + 64 + 4 * np.abs(np.where(np.isfinite(lse), lse, 0)))
    tol = size["v"] * (2.02 * u + 2 * small[:, :, None]) + SMALLEST[type] * (1 + size["sum"])
    return tol, 2 * small


def check_attend(type, d, got, got_lse, out, lse, size):
    tol, tol_lse = attend_tolerance(type, d, out, lse, size)
    served = ~np.isnan(lse)
    nothing = np.isneginf(lse) & served
    assert (got[nothing] == 0).all() and np.isneginf(got_lse[nothing]).all()
    some = served & ~nothing
    assert np.isfinite(got[some]).all() and np.isfinite(got_lse[some]).all()
    off, off_lse = np.abs(got - out)[some], np.abs(got_lse[some] - lse[some])
    assert (off <= tol[some]).all(), ("out", float((off / tol[some]).max()), float(off.max()))
    assert (off_lse <= tol_lse[some]).all(), ("lse", float((off_lse / tol_lse[some]).max()))
