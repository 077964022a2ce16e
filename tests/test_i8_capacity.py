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
