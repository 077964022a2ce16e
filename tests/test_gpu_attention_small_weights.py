"""dc_attention_paged where most weights are small beside the largest one: what many such keys add up to is in the result."""
import numpy as np
import pytest

import oracle.attention as oa
from tests.attention_cases import UNIT, SMALLEST, f64, paged
from tests.test_gpu_attention import attend

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def tolerance(type, d, lse, size):
    """Element by element, with u the unit of the type and e = 2^-24: a weight is rounded to the type once, relative u, or where it is below the
    type's normal range by at most 2^-32 of the row's largest (f16: half a step of 2^-24, beside a largest one of at least 2^7); the
    result is rounded once; a score is off by (d + 8) e of its largest sum of |q k|, sums over n keys by n e."""
    small = 2.0 ** -24 * (2 * (d + 8) * size["s"] + 2 * size["n"][:, None] + 64 + 4 * np.abs(lse))
    return size["v"] * (2.02 * UNIT[type] + 2 * small[:, :, None]) + 2.0 ** -32 * size["sum"] + SMALLEST[type], 2 * small


@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("news", [1, 20, 140])  # rows of each of the kernels
@pytest.mark.parametrize("heavy", [0, 1500, 2860])  # where the one large weight is: before the others, among them, nearly last
@pytest.mark.parametrize("power", [-15.4, -25.3, -28.0])
def test_many_small_weights_beside_a_large_one(type, d, news, heavy, power):
    length = 3000
    print(f"case small weights {type} d={d} news={news} heavy={heavy} power={power}", flush=True)
    p = paged(51, type, 1, d, 64, [length], [news])
    q = torch.zeros((news, 1, d), dtype=p["k"].dtype)
    q[:, :, 0] = 1
    low = power * float(np.log(2.0))
    for j in range(length):
        page, at = oa.place_of(p["batch"], 0, j, 64, p["n_pages"])
        p["k"][page, :, at] = 0
        p["k"][page, :, at, 0] = 0.0 if j == heavy else low
        p["v"][page, :, at] = 0.0 if j == heavy else 1.0  # only what the others add up to
    got, got_lse = attend(p, 1, q, 1.0, uniform=news == 1)
    out, lse, size = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q), 1.0)
    tol, tol_lse = tolerance(type, d, lse, size)
    off = np.abs(got - out)
    assert (off <= tol).all(), (float((off / tol).max()), float(got.flat[0]), float(out.flat[0]))
    assert (np.abs(got_lse - lse) <= tol_lse).all()


@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heavy", [0, 900])
def test_many_small_weights_in_runs_that_are_not_cut(type, d, heavy):
    """Enough sequences and heads to fill the chip: a wavefront has a quarter of a run, the large weight early among them."""
    length, n, kv = 3000, 16, 16
    print(f"case small weights uncut {type} d={d} heavy={heavy}", flush=True)
    p = paged(52, type, kv, d, 64, [length], [1])
    q = torch.zeros((n, kv, d), dtype=p["k"].dtype)
    q[:, :, 0] = 1
    for j in range(length):
        page, at = oa.place_of(p["batch"], 0, j, 64, p["n_pages"])
        p["k"][page, :, at] = 0
        p["k"][page, :, at, 0] = 0.0 if j == heavy else -25.3 * float(np.log(2.0))
        p["v"][page, :, at] = 0.0 if j == heavy else 1.0
    out, lse, size = oa.attend(f64(p["k"]), f64(p["v"]), p["batch"], f64(q[:1]), 1.0)
    many = {"lens": np.repeat(p["batch"]["lens"], n), "starts": np.arange(n + 1, dtype=np.int32), "pages": np.repeat(p["batch"]["pages"], n, 0)}
    p = dict(p, batch=dict(p["batch"], **many), news=[1] * n)  # all read the same pages
    got, got_lse = attend(p, kv, q, 1.0, uniform=True)
    tol, tol_lse = tolerance(type, d, lse, size)
    assert (np.abs(got - out) <= tol).all(), (float((np.abs(got - out) / tol).max()), float(got.flat[0]), float(out.flat[0]))
    assert (np.abs(got_lse - lse) <= tol_lse).all()
