"""How dc_attention_paged reads a common prefix when there is a window, told by its workspace (no GPU is touched: the addresses are made up):
what is joined from parts needs one, a sequence's rows that read the prefix along with their own pages in one run need none."""
import pytest

import paper_2502_15443_amd as dc

ADDR = 1 << 20


def slots(seqs, new, heads, kv_heads, prefix, own, window=0, sinks=0, d=128):
    """Parts that a row's result is joined from; 0 if it is not."""
    rows, page = seqs * new, 128
    cache = dc.KVCache(ADDR, ADDR, 100000, kv_heads, d, page, dc.TYPE_BF16)
    batch = dc.KVBatch(seqs, rows, new, prefix + own, ADDR, ADDR, -(-own // page), row_start_dev=ADDR, prefix_len=prefix,
                       prefix_pages_dev=ADDR if prefix else None)
    s = (heads * d, d)
    n = dc.attention_paged_workspace(cache, batch, dc.Attention(heads, ADDR, 2 * ADDR, None, 0.1, window=window, sinks=sinks, q_strides=s, out_strides=s))
    part = rows * heads * (d + 2) * 4
    assert n % part == 0
    return n // part


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("seqs,new,heads,kv_heads,prefix,own", [(64, 9, 32, 8, 32768, 500), (8, 40, 32, 8, 16384, 256), (4, 300, 32, 32, 1000, 700),
                                                                (12, 9, 4, 1, 7003, 50), (2, 16, 32, 8, 500, 100), (32, 1, 32, 8, 5000, 100)])
def test_a_window_that_hides_nothing_changes_nothing(d, seqs, new, heads, kv_heads, prefix, own):
    plain = slots(seqs, new, heads, kv_heads, prefix, own, d=d)
    for window in (prefix + own, 2 * (prefix + own), 2 ** 32 - 1):
        assert slots(seqs, new, heads, kv_heads, prefix, own, window, 4, d=d) == plain


def test_a_window_that_hides_most_of_the_prefix_has_it_read_along():
    # 512 workgroups of the own pages' rows fill the chip uncut: parts are joined only where the prefix is read apart
    batch = (64, 9, 32, 8, 32768, 500)
    assert slots(*batch) > 1
    assert slots(*batch, window=20000) > 1 and slots(*batch, window=20000, sinks=16) > 1
    assert slots(*batch, window=400) == 0 and slots(*batch, window=550, sinks=4) == 0
    assert slots(*batch, window=100, sinks=32768) > 1  # the first tokens, seen whatever the window, are all of it


def test_a_short_prefix_in_view_is_read_along():
    # 64 sequences of 36 rows a head behind 512 tokens: reading those once for all rows saves less than it costs to join the parts
    assert slots(64, 9, 32, 8, 512, 500) == 0
    assert slots(64, 9, 32, 8, 512, 500, window=1256) == 0 and slots(64, 9, 32, 8, 16384, 500, window=1000, sinks=12) == 0
    assert slots(64, 9, 32, 8, 16384, 500) > 1 and slots(64, 9, 32, 8, 16384, 500, window=12000) > 1
