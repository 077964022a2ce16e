"""A common prefix that many rows of each sequence read apart from the sequences' own pages.  12 sequences of 36 rows a head take 9 workgroups
more for each of 3 key/value heads than their 356 rows together; over a prefix as long as here those are estimated to cost 6 us or more, and the
join 4.5 (heads of 64) to 6 (256) at most.  With a window, what it hides of the prefix is not counted: the ones here leave nearly all of it."""
import pytest

from tests.test_gpu_attention import run

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type,d,prefix", [("bf16", 64, 7003), ("f16", 128, 5003), ("bf16", 256, 3003)])
@pytest.mark.parametrize("hides,sinks", [(None, 0), (100, 0), (300, 40), (-2 ** 31, 3)])  # by how much the window is shorter than the prefix
def test_prefix_apart(type, d, prefix, hides, sinks):
    news = [9, 1, 5, 9, 9, 9, 2, 9, 9, 0, 9, 9]
    run(81, type, 12, 3, d, 64, [prefix + n + 3 * i for i, n in enumerate(news)], news, 0 if hides is None else prefix - hides, sinks, prefix=prefix,
        absent=[(3, 0)])


def test_prefix_apart_seen_by_sinks_alone():
    news = [9, 1, 5, 9, 9, 9, 2, 9, 9, 0, 9, 9]
    run(82, "f16", 12, 3, 128, 64, [5003 + n + 3 * i for i, n in enumerate(news)], news, window=20, sinks=4800, prefix=5003)
