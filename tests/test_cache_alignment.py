"""dc_kv_append and dc_attention_paged are promised rows, tables and pools at multiples of 16 bytes: no access of their kernels may take more for granted."""
import os
import re
import subprocess

import pytest

import paper_2502_15443_amd.build as build


@pytest.mark.parametrize("name", ["dc_cache.hip", "dc_attention.hip"])
def test_no_access_takes_more_than_16_bytes_for_granted(name):
    source = os.path.join(build.PKG, "csrc", name)
    flags = [f for f in build.FLAGS if f not in ("-fPIC", "-shared", "-pthread")]
    ir = subprocess.run([build.HIPCC, *flags, "--offload-device-only", "-emit-llvm", "-S", source, "-o", "-"], check=True, capture_output=True, text=True).stdout
    accesses = re.findall(r"^.*(?:\bload |\bstore ).*\balign (\d+)", ir, re.M)
    assert len(accesses) > 100
    assert max(int(a) for a in accesses) == 16


def _rows_at(torch, x, skip):
    """x on the GPU, `skip` values behind a multiple of 32 bytes."""
    wide = torch.full((x.numel() + 32,), float("nan"), dtype=x.dtype, device="cuda")
    at = (-(wide.data_ptr() // x.element_size()) % (32 // x.element_size())) + skip
    y = wide[at:at + x.numel()].view(x.shape)
    y.copy_(x)
    assert y.data_ptr() % 32 == 16
    return y


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", ["f32", "bf16"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("d,news", [(64, [3, 1]), (128, [600, 5]), (256, [2, 2])])
def test_rows_and_tables_at_odd_multiples_of_16_bytes(x_type, neighbours, d, news):
    torch = pytest.importorskip("torch")
    import numpy as np

    import oracle.attention as oa
    import paper_2502_15443_amd as dc
    from tests.attention_cases import KIND, SMALLEST, UNIT, device_batch, device_cache, f64, paged, torch_type
    from tests.test_gpu_kv_append import angles

    print(f"case append at 16 bytes {x_type} neighbours={neighbours} d={d} news={news}", flush=True)
    heads, kv, lens, rows = 4, 2, [n + 7 for n in news], sum(news)
    p = paged(91, "bf16", kv, d, 16, lens, news, fill=7.75)
    x = {n: torch.from_numpy(p["rng"].standard_normal((rows, h, d)).astype(np.float32)).to(torch_type(x_type)) for n, h in (("k", kv), ("v", kv), ("q", heads))}
    cos, sin = (torch.from_numpy(t) for t in angles(max(lens), d // 2))
    skip = 16 // x["k"].element_size()
    kd, vd, qd = (_rows_at(torch, x[n].cuda(), skip) for n in ("k", "v", "q"))
    cd, sd = _rows_at(torch, cos.cuda(), 4), _rows_at(torch, sin.cuda(), 4)
    out = _rows_at(torch, torch.zeros((rows, heads, d), dtype=torch.bfloat16, device="cuda"), 8)
    cache, k, v = device_cache(p)
    dc.kv_append(cache, device_batch(p), dc.KVRows(KIND[x_type], heads, kd, vd, qd, out, rot_dim=d, pairing=int(neighbours), cos_dev=cd, sin_dev=sd,
                                                   n_positions=max(lens)), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    want = oa.append(f64(p["k"]), f64(p["v"]), p["batch"], f64(x["k"]), f64(x["v"]), f64(x["q"]), f64(cos), f64(sin), neighbours)
    most = max(float(t.abs().max()) for t in x.values())
    for got, w in zip((k, v, out), want):  # written once: two products and a sum in fp32, then rounded
        assert (np.abs(f64(got) - w) <= UNIT["bf16"] * np.abs(w) * 1.001 + 4 * 2.0 ** -24 * 2 * most + SMALLEST["bf16"]).all()
