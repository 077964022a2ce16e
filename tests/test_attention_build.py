"""What the build looks for in the device assembly, for the sources of the cache and the attention; and that their products are the matrix
units'."""
import importlib.util
import os
import re

import pytest

PKG = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_15443_amd")


@pytest.fixture(scope="module")
def build():
    spec = importlib.util.spec_from_file_location("dc_attention_build_checks", os.path.join(PKG, "build.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.fixture(scope="module")
def assembly(build):
    return {source: build.device_assembly(os.path.join(PKG, "csrc", source)) for source in ("dc_cache.hip", "dc_attention.hip")}


@pytest.mark.parametrize("source", ["dc_cache.hip", "dc_attention.hip"])
def test_the_builds_own_checks(build, assembly, source):
    asm = assembly[source]
    assert not build.PACKED_FP32.search(asm)
    assert build.generic_lds_addresses(asm) == [] and build.buffer_access_loops(asm) == []
    assert "flat_load" not in asm and "flat_store" not in asm


def test_sources_are_all_built(build):
    csrc = os.path.join(PKG, "csrc")
    assert sorted(os.path.basename(f) for f in build.SOURCES) == sorted(f for f in os.listdir(csrc) if f.endswith((".hip", ".cpp")))


def test_products_and_wavefronts(assembly):
    asm = assembly["dc_attention.hip"]
    assert len(re.findall(r"v_mfma_f32_32x32x16_(?:bf16|f16)", asm)) > 100 and len(re.findall(r"v_mfma_f32_16x16x32_(?:bf16|f16)", asm)) > 100
    assert "ds_read_b64_tr_b16" in asm
    # registers of a lane: 512 on a SIMD, for as many wavefronts as the kernels are written for
    most = {"dc_attention_tile_kernel": {64: 168, 128: 256, 256: 512}, "dc_attention_few_kernel": {64: 256, 128: 256, 256: 512},
            "dc_attention_both_kernel": {64: 256, 128: 256, 256: 512}}
    seen = set()
    for kernel in asm.split("amdhsa.kernels:")[1].split("\n  - ."):
        value = dict(re.findall(r"^\s*\.(\w+): +(\S+)$", kernel, re.M))
        m = re.search(r"(dc_attention_(?:tile|few|both)_kernel)I\w+?Li(\d+)", value.get("name", ""))
        if m:
            seen.add((m.group(1), int(m.group(2))))
            assert int(value["vgpr_count"]) <= most[m.group(1)][int(m.group(2))], value["name"]
            assert int(value["vgpr_spill_count"]) <= 8, value["name"]
    assert len(seen) == 9
