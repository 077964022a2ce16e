"""dc_kv_append against the oracle in 64 bits through the C ABI: types, both pairings, partial rotation, layouts, explicit positions,
ragged batches, absent pages, prefixes, and everything that must stay as it was."""
import numpy as np
import pytest

import oracle.attention as oa
import paper_2502_15443_amd as dc
from tests.attention_cases import KIND, SMALLEST, UNIT, device_batch, device_cache, f64, paged, rows_tensor, torch_type

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SENTINEL = 7.75


def angles(n, half):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(half)[None] / max(half, 1))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def run(seed, type, x_type, heads, kv_heads, d, page, lens, news, rot, neighbours, prefix=0, absent=(), layout="dense", positions=None,
        n_positions=None, uniform=False, stream=None):
    print(f"case append {x_type}->{type} heads={heads}/{kv_heads} d={d} page={page} lens={lens} news={news} rot={rot} "
          f"neighbours={neighbours} prefix={prefix} layout={layout}", flush=True)
    p = paged(seed, type, kv_heads, d, page, lens, news, prefix, absent, fill=SENTINEL)
    rows = int(p["batch"]["starts"][-1])
    x = {n: torch.from_numpy(p["rng"].standard_normal((rows, h, d)).astype(np.float32)).to(torch_type(x_type))
         for n, h in (("k", kv_heads), ("v", kv_heads), ("q", heads))}
    n_positions = n_positions or max(lens)
    cos, sin = angles(n_positions, rot // 2)
    cache, k, v = device_cache(p)
    batch = device_batch(p, uniform)
    kd, vd, qd = (rows_tensor(x[n].cuda(), layout) if x[n].shape[1] else None for n in ("k", "v", "q"))
    wide = torch.full((rows + 2, heads + 2, d), SENTINEL, dtype=torch_type(type), device="cuda")
    out = wide[1:-1, 1:-1] if heads else None
    pos_d = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda")
    cd, sd = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    r = dc.KVRows(KIND[x_type], heads, kd, vd, qd, out, rot_dim=rot, pairing=dc.ROPE_NEIGHBOURS if neighbours else dc.ROPE_HALVES,
                  cos_dev=cd if rot else None, sin_dev=sd if rot else None, n_positions=n_positions, position_dev=pos_d)
    torch.cuda.synchronize()
    dc.kv_append(cache, batch, r, torch.cuda.current_stream().cuda_stream if stream is None else stream.cuda_stream)
    torch.cuda.synchronize()
    want_k, want_v, want_q = oa.append(f64(p["k"]), f64(p["v"]), p["batch"], f64(x["k"]), f64(x["v"]), f64(x["q"]), cos.astype(np.float64),
                                       sin.astype(np.float64), neighbours, positions)
    # written once each, in fp32 and then rounded: two products and a sum of values a, b with |a|, |b| <= `most`
    most = max(float(t.abs().max()) for t in x.values() if t.numel())
    def near(got, want, what):
        tol = UNIT[type] * np.abs(want) * 1.001 + 4 * 2.0 ** -24 * 2 * most + SMALLEST[type]
        assert (np.abs(got - want) <= tol).all(), (what, float(np.abs(got - want).max()))
    near(f64(k), want_k, "k")
    # values are only rounded, and tokens that are not new are untouched
    untouched = want_k == f64(p["k"])
    assert np.array_equal(f64(k)[untouched], f64(p["k"])[untouched])
    rounded = torch.from_numpy(want_v).to(torch_type(type))
    assert torch.equal(v.cpu().view(torch.int16), rounded.view(torch.int16))
    if heads:
        got = f64(out)
        left = np.isnan(want_q)
        assert (got[left] == SENTINEL).all()
        near(got[~left], want_q[~left], "q")
        edge = wide.clone()
        edge[1:-1, 1:-1] = SENTINEL
        assert (edge == SENTINEL).all()


@pytest.mark.parametrize("type", ["bf16", "f16"])
@pytest.mark.parametrize("x_type", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("neighbours", [False, True])
def test_types_and_pairings(type, x_type, d, neighbours):
    run(1, type, x_type, 6, 2, d, 32, [40, 1, 33], [40, 1, 2], d, neighbours)


@pytest.mark.parametrize("rot", [0, 16, 32, 48, 64, 112, 128])
@pytest.mark.parametrize("neighbours", [False, True])
def test_partial_rotation(rot, neighbours):
    run(2, "bf16", "f32", 5, 5, 128, 16, [30, 17], [7, 17], rot, neighbours)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (32, 32), (40, 40), (64, 8), (71, 1), (0, 4)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_heads(heads, kv_heads, d):
    run(3, "bf16", "bf16", heads, kv_heads, d, 64, [100, 3, 65], [1, 1, 1], d, False, uniform=True)


@pytest.mark.parametrize("layout", ["heads first", "slice"])
def test_layouts(layout):
    run(4, "f16", "f16", 6, 2, 128, 16, [60, 31], [60, 5], 128, True, layout=layout)


def test_many_rows():
    # more rows than a launch of few rows has, sequences without rows among them, and more sequences than a wavefront has lanes
    run(5, "bf16", "bf16", 4, 2, 64, 16, [300, 0, 290, 7], [300, 0, 280, 0], 64, False)
    run(6, "bf16", "bf16", 2, 1, 64, 16, [1 + i % 5 for i in range(150)], [i % 2 + (i % 5 > 1) for i in range(150)], 64, False)


def test_prefix_and_absent_pages():
    run(7, "bf16", "f32", 4, 2, 64, 16, [130, 100, 75], [20, 25, 1], 32, False, prefix=70, absent=[(0, 1), (1, 1)])


def test_rows_without_a_place():
    # sequences shorter than their rows: positions below zero have no cosines, nothing is written for them
    run(8, "bf16", "bf16", 4, 2, 64, 16, [3, 0, 20], [5, 1, 2], 64, False)
    # without rotation their queries are still given
    run(9, "bf16", "bf16", 4, 2, 64, 16, [3, 0, 20], [5, 1, 2], 0, False)


def test_given_positions():
    run(10, "bf16", "bf16", 4, 2, 64, 16, [10, 20], [3, 4], 64, False, positions=[0, 5, 2, 99, 100, -1, 50], n_positions=100)


def test_another_stream():
    run(11, "bf16", "bf16", 4, 2, 128, 16, [300, 20], [300, 4], 128, False, stream=torch.cuda.Stream())


def test_queries_turned_in_place():
    p = paged(12, "bf16", 2, 128, 16, [9, 30], [4, 1], fill=SENTINEL)
    x = torch.from_numpy(p["rng"].standard_normal((5, 8, 128)).astype(np.float32)).to(torch.bfloat16)
    cos, sin = angles(30, 64)
    for neighbours in (False, True):
        cache, k, v = device_cache(p)
        rows = x.cuda()
        q, kk, vv = rows[:, :4], rows[:, 4:6], rows[:, 6:]
        r = dc.KVRows(dc.TYPE_BF16, 4, kk, vv, q, q, rot_dim=128, pairing=int(neighbours), cos_dev=torch.from_numpy(cos).cuda(),
                      sin_dev=torch.from_numpy(sin).cuda(), n_positions=30)
        dc.kv_append(cache, device_batch(p), r, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        _, _, want = oa.append(f64(p["k"]), f64(p["v"]), p["batch"], f64(x[:, 4:6]), f64(x[:, 6:]), f64(x[:, :4]), cos.astype(np.float64),
                               sin.astype(np.float64), neighbours)
        assert (np.abs(f64(q) - want) <= UNIT["bf16"] * np.abs(want) * 1.001 + 2.0 ** -21 * 5).all()
        assert torch.equal(rows[:, 4:].cpu(), x[:, 4:])


def test_replays_of_a_recorded_call():
    p = paged(13, "bf16", 2, 64, 16, [40, 30], [4, 30], fill=SENTINEL)
    x = torch.from_numpy(p["rng"].standard_normal((34, 8, 64)).astype(np.float32)).cuda()
    cos, sin = (torch.from_numpy(t).cuda() for t in angles(40, 32))
    cache, k, v = device_cache(p)
    batch = device_batch(p)
    out = torch.zeros((34, 4, 64), dtype=torch.bfloat16, device="cuda")
    r = dc.KVRows(dc.TYPE_F32, 4, x[:, 4:6], x[:, 6:], x[:, :4], out, rot_dim=64, cos_dev=cos, sin_dev=sin, n_positions=40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dc.kv_append(cache, batch, r, side.cuda_stream)
    torch.cuda.synchronize()
    want = [t.cpu().view(torch.int16).clone() for t in (k, v, out)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        dc.kv_append(cache, batch, r, side.cuda_stream)
    for _ in range(4):
        k.copy_(p["k"])
        v.copy_(p["v"])
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip((k, v, out), want):
            assert torch.equal(t.cpu().view(torch.int16), w)
