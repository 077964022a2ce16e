"""Attention over a cache of 8 bits up to the last position there is, without a window: parts of the keys begin all over the range of positions."""
import numpy as np
import pytest

import oracle.attention as oa
import oracle.cache_i8 as oc8
import paper_2502_15443_amd as dc
from tests.attention_cases import f64
from tests.i8_cases import check_attend_i8

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 2 ** 16  # positions


@pytest.mark.parametrize("d,news", [(64, 16), (128, 9), (64, 8), (128, 1)])
def test_parts_that_begin_far_behind(d, news):
    """17 to 32 rows, and up to 16, of two heads of a key/value head.  Pages are there at the beginning, where each 128th of the tiles begins and at the end."""
    print(f"case far parts d={d} news={news}", flush=True)
    page, stride = 256, MOST // 256
    entries = sorted({0, *(stride // 128 * part for part in (1, 63, 64, 65, 100, 127)), stride - 1})
    r = np.random.default_rng(5)
    n_pages = len(entries)
    k, v = (r.integers(-127, 128, (n_pages, 1, page, d)).astype(np.int8) for _ in range(2))
    ks, vs = ((2.0 ** r.integers(-7, -4, (n_pages, 1, page // 16))).astype(np.float32) for _ in range(2))
    q = torch.from_numpy(r.standard_normal((news, 2, d)).astype(np.float32)).to(torch.bfloat16)
    table = torch.full((1, stride), -1, dtype=torch.int32)
    table[0, entries] = torch.arange(n_pages, dtype=torch.int32)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    dev, qd = [torch.from_numpy(x.copy()).cuda() for x in (k, v, ks, vs)], q.cuda()
    cache = dc.KVCache(dev[0], dev[1], n_pages, 1, d, page, dc.TYPE_I8, scale_tokens=16, k_scale_dev=dev[2], v_scale_dev=dev[3])
    batch = dc.KVBatch(1, news, news, MOST, i32([MOST]), table.cuda(), stride, row_start_dev=i32([0, news]))
    out, lse = torch.empty_like(qd), torch.empty((news, 2), dtype=torch.float32, device="cuda")
    a = dc.Attention(2, qd, out, lse, d ** -0.5)
    n = dc.attention_paged_workspace(cache, batch, a)
    dc.attention_paged(cache, batch, a, torch.empty(n + 16, dtype=torch.uint8, device="cuda"), n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    short = {"lens": [n_pages * page], "starts": [0, news], "pages": np.arange(n_pages)[None], "prefix_len": 0, "prefix_pages": []}
    want = oa.attend(oc8.values(k, ks), oc8.values(v, vs), short, f64(q), np.float64(np.float32(d ** -0.5)))
    check_attend_i8("bf16", d, f64(out), f64(lse), *want, 2.0 ** -5)
