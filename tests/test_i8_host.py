"""Host side of the cache of 8 bits and of dc_kv_tables: what is refused before anything is enqueued (no GPU is touched: the addresses are made up), what
the workspace calls say, and pins of the oracles."""
import numpy as np
import pytest

import oracle.cache_i8 as oc8
import oracle.tables as ot
import paper_2502_15443_amd as dc
from tests.test_attention_host import attention, batch, refused, rows

ADDR = 1 << 20
E_ARG, E_CAP = -1, -2


def cache(**kw):
    c = dc.KVCache(ADDR, ADDR, 10, 2, 128, 64, dc.TYPE_I8, rows_type=dc.TYPE_F16, scale_tokens=32, k_scale_dev=ADDR + 4, v_scale_dev=ADDR)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def requests(**kw):
    q = dc.KVRequests(3, 20, 16, 7, 100, held_dev=ADDR, new_dev=ADDR, pages_in_dev=ADDR, queue_in_dev=ADDR, free_dev=ADDR, len_dev=ADDR, row_start_dev=ADDR,
                      pages_dev=ADDR, queue_dev=ADDR, slot_dev=ADDR, position_dev=ADDR, seq_dev=ADDR)
    for k, v in kw.items():
        setattr(q, k, v)
    return q


BAD_CACHE = [dict(type=2), dict(type=4), dict(rows_type=2), dict(rows_type=3), dict(rows_type=7), dict(scale_tokens=0), dict(scale_tokens=1), dict(scale_tokens=8),
             dict(scale_tokens=48), dict(scale_tokens=128), dict(scale_tokens=256), dict(scale_tokens=2 ** 31), dict(k_scale_dev=None), dict(v_scale_dev=None),
             dict(k_scale_dev=ADDR + 2), dict(v_scale_dev=ADDR + 1), dict(head_dim=96), dict(head_dim=32), dict(page_tokens=8), dict(page_tokens=16),
             dict(n_kv_heads=0), dict(n_pages=0), dict(n_pages=2 ** 31), dict(k_dev=None), dict(v_dev=None), dict(k_dev=ADDR + 8), dict(v_dev=ADDR + 1)]
BAD_REQUESTS = [dict(n_seqs=0), dict(n_seqs=65536), dict(n_rows=0), dict(n_rows=2 ** 24), dict(page_tokens=0), dict(page_tokens=8), dict(page_tokens=24),
                dict(page_tokens=512), dict(pages_stride=0), dict(pages_stride=2 ** 27), dict(n_pages=0), dict(n_pages=2 ** 31), dict(prefix_len=5),
                dict(prefix_pages_dev=ADDR), dict(prefix_len=2 ** 31 - 2 ** 16 - 96, prefix_pages_dev=ADDR), dict(slot_dev=ADDR + 4), dict(position_dev=ADDR + 2),
                dict(seq_dev=ADDR + 1), dict(prefix_len=3, prefix_pages_dev=ADDR + 2)] + \
    [{n: bad} for n in ("held_dev", "new_dev", "pages_in_dev", "queue_in_dev", "free_dev", "len_dev", "row_start_dev", "pages_dev", "queue_dev") for bad in (None, ADDR + 2)]


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_caches_that_are_refused(bad):
    refused(E_ARG, dc.kv_append, cache(**bad), batch(), rows())
    refused(E_ARG, dc.attention_paged_workspace, cache(**bad), batch(), attention())
    refused(E_ARG, dc.attention_paged, cache(**bad), batch(), attention(), ADDR, 1 << 40)


def test_batches_rows_and_attentions_are_checked_too():
    from tests.test_attention_host import BAD_ATTENTION, BAD_BATCH, BAD_ROWS

    for bad in BAD_BATCH:
        if "pages_stride" in bad or "prefix_len" in bad:
            continue  # sized for pages of 16 tokens
        refused(E_ARG, dc.kv_append, cache(), batch(**bad), rows())
        refused(E_ARG, dc.attention_paged, cache(), batch(**bad), attention(), ADDR, 1 << 40)
    for bad in BAD_ROWS:
        if bad.get("type") != dc.TYPE_F16:
            refused(E_ARG, dc.kv_append, cache(), batch(), rows(**bad))
    for bad in BAD_ATTENTION:
        refused(E_ARG, dc.attention_paged, cache(), batch(), attention(**bad), ADDR, 1 << 40)


def test_queries_in_place_are_of_the_rows_type():
    # bf16 rows turned in place, of a cache whose queries are f16
    refused(E_ARG, dc.kv_append, cache(), batch(), rows(q_dev=2 * ADDR))


def test_the_fields_of_a_cache_of_8_bits_are_not_read_for_the_others():
    c = dc.KVCache(ADDR, ADDR, 10, 2, 128, 64, dc.TYPE_BF16)
    c.rows_type, c.scale_tokens, c.k_scale_dev = 99, 7, 3
    assert dc.attention_paged_workspace(c, batch(), attention()) == dc.attention_paged_workspace(dc.KVCache(ADDR, ADDR, 10, 2, 128, 64), batch(), attention())


def test_small_workspaces_are_refused():
    c, b, a = cache(), batch(max_len=100000, pages_stride=2000), attention()
    n = dc.attention_paged_workspace(c, b, a)
    assert n > 0
    refused(E_CAP, dc.attention_paged, c, b, a, ADDR, n - 1)
    refused(E_ARG, dc.attention_paged, c, b, a, None, n)
    refused(E_ARG, dc.attention_paged, c, b, a, ADDR + 8, n)
    q = requests()
    n = dc.kv_tables_workspace(q)
    refused(E_CAP, dc.kv_tables, q, ADDR, n - 1)
    refused(E_ARG, dc.kv_tables, q, None, n)
    refused(E_ARG, dc.kv_tables, q, ADDR + 8, n)


@pytest.mark.parametrize("bad", BAD_REQUESTS, ids=str)
def test_requests_that_are_refused(bad):
    refused(E_ARG, dc.kv_tables_workspace, requests(**bad))
    refused(E_ARG, dc.kv_tables, requests(**bad), ADDR, 1 << 40)


def test_requests_at_their_limits():
    refused(E_ARG, dc.kv_tables_workspace, requests(n_seqs=65535, pages_stride=32769))
    assert dc.kv_tables_workspace(requests(n_seqs=65535, pages_stride=32768)) > 65535 * 16
    assert dc.kv_tables_workspace(requests(n_seqs=1, pages_stride=(2 ** 31 - 2 ** 16) // 16)) > 0
    refused(E_ARG, dc.kv_tables, None, ADDR, 1 << 40)


def test_oracle_scales():
    for most, s in ((0.0, 2.0 ** -126), (127.0, 1.0), (127.00001, 2.0), (63.5, 0.5), (64.0, 1.0), (3.4028234e38, 2.0 ** 122), (1e-45, 2.0 ** -126)):
        assert oc8.scale_for(np.float32(most)) == np.float32(s), most
    assert [oc8.sound(s) for s in (np.nan, -1.0, 0.0, 0.5)] == [2.0 ** -126, 2.0 ** -126, 2.0 ** -126, 0.5]
    assert oc8.whole([0.5, 1.5, -2.5, 200, np.inf, -np.inf, np.nan], 1.0).tolist() == [0, 2, -2, 127, 127, -127, 0]


def test_oracle_append_by_hand():
    k, v = np.full((2, 1, 16, 64), 99, np.int8), np.full((2, 1, 16, 64), 99, np.int8)
    ks, vs = np.full((2, 1, 1), 1.0, np.float32), np.full((2, 1, 1), np.nan, np.float32)
    b = {"lens": [17], "starts": [0, 2], "pages": np.array([[1, 0]]), "prefix_len": 0, "prefix_pages": []}
    x = np.zeros((2, 1, 64), np.float32)
    x[0, 0, 0], x[1, 0, 0] = 200.0, 3.0  # places 15 of page 1 and 0 of page 0
    k2, v2, ks2, vs2 = oc8.append(k, v, ks, vs, b, 16, x, x, None, None, False)
    assert ks2[1, 0, 0] == 2.0 and (k2[1, 0, :15] == 50).all() and k2[1, 0, 15, 0] == 100 and k2[0, 0, 0, 0] == 96 and ks2[0, 0, 0] == 2.0 ** -5
    assert vs2[1, 0, 0] == 2.0 and (v2[1, 0, :15] == 0).all() and (k2[0, 0, 1:] == 99).all()


def test_oracle_tables_by_hand():
    r = ot.tables([17, 5, 40], [16, 0, -1], [[3, 7, -1], [5, -1, -1], [0, 1, 2]], [9, 8, 6, 4, -1, -1, -1, -1, -1, -1], (0, 1), 18, 16, 10)
    assert r["pages"] == [[3, 7, 9], [5, -1, -1], [-1, -1, -1]] and r["queue"] == [1, 3, 0] and r["free"] == [9, 0, 1, 2, -1, -1, -1, -1, -1, -1]
    assert r["lens"] == [33, 5, 0] and r["starts"] == [0, 16, 16, 16]
    assert r["slots"] == [7 * 16 + i for i in range(1, 16)] + [9 * 16, -1, -1] and r["positions"][:2] == [17, 18] and r["seqs"][15:] == [0, -1, -1]
