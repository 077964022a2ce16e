"""How large a batch over a cache of 8 bits may be: what is beyond the limits is refused before anything is enqueued (no GPU is touched: the addresses are
made up)."""
import pytest

import paper_2502_15443_amd as dc

ADDR = 1 << 20


def problem(heads, kv_heads, d, seqs, rows, max_new, prefix=0, max_len=100):
    cache = dc.KVCache(ADDR, ADDR, 10, kv_heads, d, 16, dc.TYPE_I8, scale_tokens=16, k_scale_dev=ADDR, v_scale_dev=ADDR)
    batch = dc.KVBatch(seqs, rows, max_new, max_len + prefix, ADDR, ADDR, 7, row_start_dev=ADDR, prefix_len=prefix, prefix_pages_dev=ADDR if prefix else None)
    strides = (heads * d, d)
    return cache, batch, dc.Attention(heads, ADDR, 2 * ADDR, None, 0.1, q_strides=strides, out_strides=strides)


def refused(cache, batch, attention):
    for call in (lambda: dc.attention_paged_workspace(cache, batch, attention), lambda: dc.attention_paged(cache, batch, attention, ADDR, 1 << 60)):
        with pytest.raises(dc.DCError) as e:
            call()
        assert e.value.code == -1


@pytest.mark.parametrize("prefix", [0, 40])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_too_many_rows_of_many_sequences_are_refused(d, prefix):
    """Sequences of more rows than are few, times key/value heads, beyond 2^24."""
    refused(*problem(32768, 32768, d, 600, 1000, 40, prefix))
    refused(*problem(65535, 65535, d, 300, 32000, 300, prefix))


def test_more_threads_than_a_launch_may_have_are_refused():
    """Both ways, by 256 rows a workgroup and by 128; and nothing is refused that 128 do."""
    refused(*problem(65535, 65535, 128, 257, 1000, 140))
    for seqs in (127, 128, 129, 240):
        cache, batch, attention = problem(65535, 65535, 128, seqs, 1000, 140)
        dc.attention_paged_workspace(cache, batch, attention)


@pytest.mark.gpu
@pytest.mark.parametrize("seqs", [128, 129])
def test_as_many_workgroups_as_a_launch_has_room_for(seqs):
    """65535 heads times 128 sequences, most of them without rows: 2^32 threads of workgroups of 256 rows, with or without those of few rows."""
    torch = pytest.importorskip("torch")
    import numpy as np

    import oracle.attention as oa
    import oracle.cache_i8 as oc8
    from tests.attention_cases import f64
    from tests.i8_cases import check_attend_i8

    print(f"case as many workgroups as there may be, {seqs} sequences", flush=True)
    heads, d, page, rows = 65535, 128, 16, 160
    news = [140] + [1] * 19 + [0] * (seqs - 21) + [1]
    lens = [n + 7 for n in news]
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    stride = -(-max(lens) // page)
    table = np.arange(seqs * stride, dtype=np.int32).reshape(seqs, stride) % 2
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randint(-127, 128, (2, heads, page, d), generator=g, device="cuda", dtype=torch.int8) for _ in range(2))
    ks, vs = (2.0 ** torch.randint(-7, -4, (2, heads, 1), generator=g, device="cuda").float() for _ in range(2))
    q = torch.randn((rows, d), generator=g, device="cuda").to(torch.bfloat16)
    out, lse = torch.full((rows, heads, d), 7.75, device="cuda", dtype=torch.bfloat16), torch.full((rows, heads), 7.75, device="cuda")
    i32 = lambda x: torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()  # noqa: E731
    cache = dc.KVCache(k, v, 2, heads, d, page, dc.TYPE_I8, scale_tokens=16, k_scale_dev=ks, v_scale_dev=vs)
    batch = dc.KVBatch(seqs, rows, 140, max(lens), i32(lens), i32(table), stride, row_start_dev=i32(starts))
    a = dc.Attention(heads, q, out, lse, d ** -0.5, q_strides=(d, 0))
    n = dc.attention_paged_workspace(cache, batch, a)
    dc.attention_paged(cache, batch, a, torch.empty(n + 16, dtype=torch.uint8, device="cuda"), n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    some = [0, 1, 2 ** 15, heads - 2, heads - 1]
    pools = [oc8.values(x[:, some].cpu().numpy(), s[:, some].cpu().numpy()) for x, s in ((k, ks), (v, vs))]
    want = oa.attend(*pools, {"lens": lens, "starts": starts, "pages": table, "prefix_len": 0, "prefix_pages": []},
                     f64(q)[:, None].repeat(len(some), 1), np.float64(np.float32(d ** -0.5)))
    check_attend_i8("bf16", d, f64(out[:, some]), f64(lse[:, some]), *want, 2.0 ** -5)
