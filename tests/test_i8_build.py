"""What the build looks for in the device assembly, for the sources of the cache of 8 bits and of the tables: that products are the matrix units', that no access takes
more than 16 bytes for granted, and that kernels have the registers that they are written for."""
import re
import subprocess

import pytest

import paper_2502_15443_amd.build as build
from tests.test_attention_build import PKG

SOURCES = ["dc_cache_i8.hip", "dc_attention_i8.hip", "dc_tables.hip"]


@pytest.fixture(scope="module")
def assembly():
    return {source: build.device_assembly(f"{PKG}/csrc/{source}") for source in SOURCES}


@pytest.mark.parametrize("source", SOURCES)
def test_the_builds_own_checks(assembly, source):
    asm = assembly[source]
    assert not build.PACKED_FP32.search(asm)
    assert build.generic_lds_addresses(asm) == [] and build.buffer_access_loops(asm) == []
    assert "flat_load" not in asm and "flat_store" not in asm


def test_products_and_wavefronts(assembly):
    asm = assembly["dc_attention_i8.hip"]
    assert len(re.findall("v_mfma_f32_32x32x16_f16", asm)) > 100 and len(re.findall("v_mfma_f32_16x16x32_f16", asm)) > 100
    assert "ds_read_b64_tr_b8" in asm and "ds_read_b64_tr_b16" in asm
    # registers of a lane: 512 on a SIMD, for as many wavefronts as the kernels are written for
    most = {"tile": {64: 168, 128: 256, 256: 512}, "few": {64: 256, 128: 256, 256: 512}, "both": {64: 256, 128: 256, 256: 512}}
    seen = set()
    for kernel in asm.split("amdhsa.kernels:")[1].split("\n  - ."):
        value = dict(re.findall(r"^\s*\.(\w+): +(\S+)$", kernel, re.M))
        m = re.search(r"dc_attention_i8_(tile|few|both)_kernelI\w+?Li(\d+)", value.get("name", ""))
        if m:
            seen.add((m.group(1), int(m.group(2))))
            assert int(value["vgpr_count"]) <= most[m.group(1)][int(m.group(2))], value["name"]
            assert int(value["vgpr_spill_count"]) <= 8, value["name"]
    assert len(seen) == 9


@pytest.mark.parametrize("source", SOURCES[:2])
def test_no_access_takes_more_than_16_bytes_for_granted(source):
    flags = [f for f in build.FLAGS if f not in ("-fPIC", "-shared", "-pthread")]
    ir = subprocess.run([build.HIPCC, *flags, "--offload-device-only", "-emit-llvm", "-S", f"{PKG}/csrc/{source}", "-o", "-"], check=True, capture_output=True,
                        text=True).stdout
    accesses = re.findall(r"^.*(?:\bload |\bstore ).*\balign (\d+)", ir, re.M)
    assert len(accesses) > 100
    assert max(int(a) for a in accesses) == 16
