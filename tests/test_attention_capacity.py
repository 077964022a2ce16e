"""How many positions a batch may have: the kernels' positions are 32-bit numbers with room for a few tiles more."""
import pytest

import paper_2502_15443_amd as dc

ADDR = 1 << 20
MOST = 2 ** 31 - 2 ** 16  # prefix_len + pages_stride * page_tokens


@pytest.mark.parametrize("page", [16, 128, 256])
@pytest.mark.parametrize("prefix", [0, 256, 2 ** 30])
def test_positions_beyond_the_limit_are_refused(page, prefix):
    cache = dc.KVCache(ADDR, ADDR, 10, 2, 128, page, dc.TYPE_BF16)
    s = (512, 128)
    a = dc.Attention(4, ADDR, 2 * ADDR, None, 0.1, q_strides=s, out_strides=s, window=100)
    r = dc.KVRows(dc.TYPE_BF16, 4, ADDR, ADDR, ADDR, 2 * ADDR, k_strides=s, v_strides=s, q_strides=s, q_out_strides=s)
    for over in (1, 2 ** 16 // page - 1):
        batch = dc.KVBatch(1, 1, 1, 100, ADDR, ADDR, (MOST - prefix) // page + over, prefix_len=prefix, prefix_pages_dev=ADDR if prefix else None)
        for call in (lambda: dc.attention_paged_workspace(cache, batch, a), lambda: dc.attention_paged(cache, batch, a, ADDR, 1 << 40),
                     lambda: dc.kv_append(cache, batch, r)):
            with pytest.raises(dc.DCError) as e:
                call()
            assert e.value.code == -1
    batch = dc.KVBatch(1, 1, 1, 100, ADDR, ADDR, (MOST - prefix) // page, prefix_len=prefix, prefix_pages_dev=ADDR if prefix else None)
    dc.attention_paged_workspace(cache, batch, a)


@pytest.mark.parametrize("rows,seqs,heads,kv_heads,good", [(2 ** 23, 1, 255, 1, True), (2 ** 23, 1, 256, 1, False), (65535, 65535, 256, 256, True),
                                                           (65535, 65535, 257, 257, False)])
def test_batches_that_are_too_large_are_refused(rows, seqs, heads, kv_heads, good):
    cache = dc.KVCache(ADDR, ADDR, 10, kv_heads, 64, 16, dc.TYPE_BF16)
    batch = dc.KVBatch(seqs, rows, rows // seqs, 100, ADDR, ADDR, 7, row_start_dev=ADDR)
    a = dc.Attention(heads, ADDR, 2 * ADDR, None, 0.1, q_strides=(heads * 64, 64), out_strides=(heads * 64, 64))
    if good:
        dc.attention_paged_workspace(cache, batch, a)
        return
    for call in (lambda: dc.attention_paged_workspace(cache, batch, a), lambda: dc.attention_paged(cache, batch, a, ADDR, 1 << 40)):
        with pytest.raises(dc.DCError) as e:
            call()
        assert e.value.code == -1


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("news,window,sinks", [(1, 100, 0), (20, 300, 5), (200, 64, 0), (150, 1, 20)])
def test_the_last_positions_there_are(d, news, window, sinks):
    """A sequence that ends at the last position, through a window; all pages but the first and the last ones have been given back."""
    torch = pytest.importorskip("torch")
    import numpy as np

    import oracle.attention as oa
    from tests.attention_cases import KIND, check_attend, f64

    print(f"case last positions d={d} news={news} window={window} sinks={sinks}", flush=True)
    page, stride, kept = 256, MOST // 256, 3
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn((kept + 1, 1, page, d), generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((news, 2, d), generator=g).to(torch.bfloat16)
    table = torch.full((1, stride), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = kept
    table[0, -kept:] = torch.arange(kept, dtype=torch.int32)
    kd, vd, qd = k.cuda(), v.cuda(), q.cuda()
    cache = dc.KVCache(kd, vd, kept + 1, 1, d, page, KIND["bf16"])
    batch = dc.KVBatch(1, news, news, MOST, torch.tensor([MOST], dtype=torch.int32, device="cuda"), table, stride,
                       row_start_dev=torch.tensor([0, news], dtype=torch.int32, device="cuda"))
    out, lse = torch.empty_like(qd), torch.empty((news, 2), dtype=torch.float32, device="cuda")
    a = dc.Attention(2, qd, out, lse, d ** -0.5, window=window, sinks=sinks)
    n = dc.attention_paged_workspace(cache, batch, a)
    dc.attention_paged(cache, batch, a, torch.empty(n + 16, dtype=torch.uint8, device="cuda"), n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    # the same rows in a sequence without the pages between: positions keep their distances from one another, and the sinks are in front
    short = {"lens": [(kept + 1) * page], "starts": [0, news], "pages": np.array([[kept, *range(kept)]]), "prefix_len": 0, "prefix_pages": []}
    want = oa.attend(f64(k), f64(v), short, f64(q), np.float64(np.float32(d ** -0.5)), window, sinks)
    check_attend("bf16", d, f64(out), f64(lse), *want)
