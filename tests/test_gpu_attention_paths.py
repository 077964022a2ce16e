"""dc_attention_paged where its kernels meet: numbers of rows at which another kernel is taken, prefixes read apart, along with the
sequences' own pages or in one launch with them, runs of keys cut in many parts, and tiles beyond the sixteen that are looked up at once."""
import numpy as np
import pytest

import oracle.attention as oa
from tests.attention_cases import check_attend, f64, paged
from tests.test_gpu_attention import attend, queries, run

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows", [16, 17, 32, 33, 128, 129, 257])
def test_numbers_of_rows(d, rows):
    # as heads of one token, and as tokens of one head
    run(31, "bf16", rows, 1, d, 16, [77, 130], [1, 1], uniform=True)
    run(32, "f16", 1, 1, d, 16, [rows + 40, rows], [rows, 1])


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 5), (1200, 70)])
def test_long_runs_of_keys(type, d, window, sinks):
    # many tiles to a workgroup, and many parts to a run; the second sequence is short, so that most of its parts see nothing
    run(33, type, 3, 1, d, 32, [2600, 90], [1, 1], window, sinks, uniform=True)
    run(34, type, 2, 1, d, 64, [2600, 90], [150, 60], window, sinks)


def test_one_long_run_with_pages_missing():
    absent = [(0, i) for i in range(0, 150, 7)] + [(0, i) for i in range(64, 90)]
    run(35, "bf16", 4, 1, 128, 16, [2500], [1], absent=absent, uniform=True)
    run(36, "bf16", 2, 1, 128, 16, [2500], [140], absent=absent)
    run(37, "bf16", 2, 1, 64, 16, [2500], [140], window=700, sinks=100, absent=absent)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("prefix", [16, 130, 1100])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 33)])
def test_prefix_along_with_the_own_pages(d, prefix, window, sinks):
    run(38, "bf16", 4, 2, d, 16, [prefix + 200, prefix + 70, prefix + 64], [150, 70, 64], window, sinks, prefix=prefix)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("prefix", [40, 700])
def test_prefix_apart_from_the_own_pages(d, prefix):
    # 12 sequences of 36 rows a head: their prefix is read by all of them together, in four workgroups instead of twelve
    news = [9, 1, 5, 9, 9, 9, 2, 9, 9, 0, 9, 9]
    run(39, "f16", 4, 1, d, 16, [prefix + n + 3 * i for i, n in enumerate(news)], news, prefix=prefix)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_long_prefix_apart_from_the_own_pages(d):
    # twelve workgroups instead of three over a prefix of this length cost more than what is joined afterwards
    news = [9, 1, 5, 9, 9, 9, 2, 9, 9, 0, 9, 9]
    run(44, "bf16", 4, 1, d, 64, [7003 + n + 3 * i for i, n in enumerate(news)], news, prefix=7003, absent=[(3, 0)])


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(9, 1), (40, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (260, 4)])
def test_prefix_and_own_pages_in_one_launch(d, heads, kv_heads, window, sinks):
    lens = [540 + 17 * i for i in range(20)]
    run(40, "bf16", heads, kv_heads, d, 32, lens, [1] * 20, window, sinks, prefix=500, uniform=True)


def test_batches_with_sequences_that_bring_nothing():
    news = [0] * 70 + [3] + [0] * 64 + [40, 1, 0]
    run(41, "bf16", 4, 2, 64, 16, [n + 2 for n in news], news)
    run(42, "bf16", 2, 1, 64, 16, [22 + n for n in news], news, prefix=21)


@pytest.mark.parametrize("news,kv_heads", [([130, 30], 1), ([5, 3], 1), ([9] * 12, 1), ([2] * 24, 2)])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_values_that_are_no_numbers_behind_a_prefix(news, kv_heads, value):
    """In the prefix and behind it, at tokens that some rows see and others do not: results that see one are no numbers, others exact."""
    prefix, window, heads, d = 75, 45, 4, 128
    lens = [prefix + n + 20 for n in news]
    p = paged(43, "bf16", kv_heads, d, 16, lens, news, prefix)
    q = queries(p, heads, "bf16")
    bad = [(0, 1, 3), (0, 60, 8), (0, prefix + 2, 21), (len(news) - 1, lens[-1] - 1, 90), (0, lens[0] - 1, 127)]  # sequence, position, value
    for b, j, i in bad:
        page, at = oa.place_of(p["batch"], b, j, 16, p["n_pages"])
        p["v"][page, 0, at, i] = value
    got, got_lse = attend(p, heads, q, 0.1, window, 2)
    clean = p["v"].nan_to_num(0.0, 0.0, 0.0)
    out, lse, size = oa.attend(f64(p["k"]), f64(clean), p["batch"], f64(q), np.float64(np.float32(0.1)), window, 2)
    mark = np.zeros(out.shape, dtype=bool)
    for b, j, i in bad:
        for s in range(len(news)):
            if j < prefix or s == b:
                for row in range(int(p["batch"]["starts"][s]), int(p["batch"]["starts"][s + 1])):
                    pos = lens[s] - (int(p["batch"]["starts"][s + 1]) - row)
                    if j <= pos and (j > pos - window or j < 2):
                        mark[row, :heads // kv_heads, i] = True
    assert mark.any() and not mark.all()
    assert not np.isfinite(got[mark]).any()
    check_attend("bf16", d, np.where(mark, out, got), got_lse, out, lse, size)


def test_rows_whose_scores_are_no_numbers_or_infinite():
    """A row that sees only NaN scores is NaN; one whose scores are all minus infinity counts as seeing nothing."""
    for news in (1, 40):
        p = paged(44, "bf16", 1, 64, 16, [news + 3, news + 3], [news, news])
        q = torch.ones((2 * news, 1, 64), dtype=torch.bfloat16)
        for b, value in ((0, float("nan")), (1, float("-inf"))):
            for j in range(news + 3):
                page, at = oa.place_of(p["batch"], b, j, 16, p["n_pages"])
                p["k"][page, 0, at, 7] = value
        got, got_lse = attend(p, 1, q, 0.5)
        assert np.isnan(got[:news]).all() and np.isnan(got_lse[:news]).all()
        assert (got[news:] == 0).all() and np.isneginf(got_lse[news:]).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("news,length", [(1, 4), (1, 700), (40, 43), (40, 1500)])
def test_rows_whose_scores_are_all_minus_infinity_beside_infinite_values(d, news, length):
    """Such rows count as seeing nothing, whatever the values are."""
    p = paged(45, "f16", 1, d, 16, [length, length], [news, news])
    q = torch.ones((2 * news, 1, d), dtype=torch.float16)
    for b in (0, 1):
        for j in range(length):
            page, at = oa.place_of(p["batch"], b, j, 16, p["n_pages"])
            p["k"][page, 0, at, 7] = float("-inf")
            if b == 0:
                p["v"][page, 0, at, j % d] = float("inf")
    got, got_lse = attend(p, 1, q, 0.1)
    assert (got == 0).all() and np.isneginf(got_lse).all()
