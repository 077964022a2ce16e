"""Attention over a cache of 8 bits whose value scales lie very far apart: a row's result depends on the scales of the blocks that it sees, and on no others,
however much larger those are.  Later tokens of the same tile, tokens that only earlier rows' windows reach, tokens of a common prefix that only another
sequence's rows see; few and many rows, and both kinds in one batch.

A result is checked by the largest scale among the blocks of which its row sees a token (not by the largest there is)."""
import numpy as np
import pytest

import oracle.attention as oa
from oracle.cache_i8 import sound
from tests.attention_cases import f64
from tests.i8_cases import check_attend_i8, paged_i8, pool_values

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def largest_scales(p, heads, window, sinks):
    """[rows, heads, 1]: the largest value scale of the blocks that a row sees a token of."""
    batch, scales = p["batch"], p["vs"]
    out = np.zeros((int(batch["starts"][-1]), heads, 1))
    group = heads // p["kv_heads"]
    for b, length in enumerate(batch["lens"]):
        first, end = int(batch["starts"][b]), int(batch["starts"][b + 1])
        at = [oa.place_of(batch, b, j, p["page"], p["n_pages"]) for j in range(int(length))]
        of = np.array([[0.0] * p["kv_heads"] if w is None else [sound(scales[w[0], h, w[1] // p["block"]]) for h in range(p["kv_heads"])] for w in at])
        for row in range(first, end):
            pos = int(length) - (end - row)
            j = np.arange(int(length))
            sees = (j <= pos) & ((j > pos - window) | (j < sinks) if window else True)
            if sees.any():
                out[row, :, 0] = np.repeat(of[sees].max(axis=0), group)
    return out


def run(type, heads, kv_heads, d, page, block, lens, news, scales, window=0, sinks=0, prefix=0, uniform=False, seed=1, change=None):
    from tests.test_gpu_attention_i8 import attend, queries

    print(f"case scales of rows {type} heads={heads}/{kv_heads} d={d} page={page} block={block} lens={lens} news={news} scales={scales} window={window} "
          f"sinks={sinks} prefix={prefix}", flush=True)
    p = paged_i8(seed, kv_heads, d, page, block, lens, news, prefix, rows_type=type, scales=scales)
    p["ks"] = np.where(np.isfinite(p["ks"]) & (p["ks"] > 0) & (p["ks"] < 1e38), 2.0 ** -5, p["ks"]).astype(np.float32)  # scores are ordinary ones
    if change:
        change(p)
    q = queries(p, heads)
    got, got_lse = attend(p, heads, q, d ** -0.5, window, sinks, uniform=uniform)
    want = oa.attend(*pool_values(p), p["batch"], f64(q), np.float64(np.float32(d ** -0.5)), window, sinks)
    check_attend_i8(type, d, got, got_lse, *want, largest_scales(p, heads, window, sinks))


# rows of a workgroup: 16 and 32, which few rows are, 128 and 256; sequences of both kinds in a batch
ROWS = [(2, 1, [7, 8, 3]), (8, 1, [4, 2, 1]), (4, 2, [150, 40]), (2, 2, [300]), (4, 1, [130, 1, 4, 2])]


@pytest.mark.parametrize("scales", [(-40, 40), (-118, 100), (-126, -95)])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,news", ROWS)
def test_blocks_of_later_tokens(heads, kv_heads, news, d, scales):
    run("bf16", heads, kv_heads, d, 16, 16, [n + 150 for n in news], news, scales)
    run("bf16", heads, kv_heads, d, 32, 16, news, news, scales, seed=2)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,news", ROWS)
@pytest.mark.parametrize("window,sinks", [(5, 0), (33, 3), (100, 20)])
def test_blocks_behind_the_window(heads, kv_heads, news, window, sinks, d):
    run("bf16", heads, kv_heads, d, 16, 16, [n + 150 for n in news], news, (-60, 60), window, sinks)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,news", ROWS + [(8, 2, [1] * 40)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 2)])
def test_blocks_of_a_prefix_that_other_sequences_see(heads, kv_heads, news, window, sinks, d):
    lens = [100 + n + 11 * i for i, n in enumerate(news)]  # the further sequences' windows leave less and less of the prefix
    run("bf16", heads, kv_heads, d, 16, 16, lens, news, (-60, 60), window, sinks, prefix=100, uniform=len(news) == 40)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,news", ROWS)
def test_one_block_far_above_the_others(heads, kv_heads, news, d):
    """The block of the sequence's last 16 tokens at 2^100; f16 results of the rows before it are of ordinary size."""
    def change(p):
        for b, n in enumerate(p["batch"]["lens"]):
            page, at = oa.place_of(p["batch"], b, int(n) - 1, p["page"], p["n_pages"])
            p["vs"][page, :, at // p["block"]] = 2.0 ** 100

    run("bf16", heads, kv_heads, d, 16, 16, [n + 150 for n in news], news, (-6, -4), change=change)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,news", ROWS + [(8, 2, [1] * 40)])
@pytest.mark.parametrize("prefix", [97, 101, 111])
def test_the_end_of_the_prefix(heads, kv_heads, news, prefix, d):
    """The prefix ends inside its last block, whose scale is 2^100; rows' windows begin before, in and behind that block, and where its 16 tokens would end."""
    def change(p):
        p["vs"][p["batch"]["prefix_pages"][-1], :, 0] = 2.0 ** 100

    lens = [prefix + n + i % 40 for i, n in enumerate(news)]
    for window, sinks in ((5, 0), (20, 0), (33, 97), (33, 98)):
        run("bf16", heads, kv_heads, d, 16, 16, lens, news, (-6, -4), window, sinks, prefix=prefix, uniform=len(news) == 40, change=change)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("news", [[1], [9], [150]])
def test_the_smallest_scales(news, d):
    """All of a sequence's values at the smallest scale there is."""
    run("bf16", 2, 1, d, 16, 16, [300], news, (-126, -126))
