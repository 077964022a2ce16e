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


def test_registers_of_the_kernels_for_mixed_batches_and_of_the_append(assembly):
    """No vector register goes to memory, but for one of heads of 64, of which three workgroups share a compute unit; scalar ones that do not fit are lanes of at most two."""
    most = {64: 168, 128: 256, 256: 512}
    seen = {"mixed": 0, "rows": 0, "blocks": 0, "both": 0}
    for source in SOURCES[:2]:
        for kernel in assembly[source].split("amdhsa.kernels:")[1].split("\n  - ."):
            value = dict(re.findall(r"^\s*\.(\w+): +(\S+)$", kernel, re.M))
            m = re.search(r"dc_(attention|kv_append)_i8_(mixed|rows|blocks|both)_kernelI\w+?Li(\d+)(?:ELb[01]ELi(\d))?", value.get("name", ""))
            if not m or (m.group(1) == "attention") != (m.group(2) == "mixed"):
                continue
            seen[m.group(2)] += 1
            # the append's blocks that are a workgroup's (rows to a thread: 0) have up to 1024 threads
            limit = most[int(m.group(3))] if m.group(2) == "mixed" else 128 if m.group(4) == "0" else 256
            assert int(value["vgpr_count"]) <= limit, value["name"]
            assert int(value["vgpr_spill_count"]) <= (1 if m.group(2) == "mixed" and m.group(3) == "64" else 0), value["name"]
            assert int(value["sgpr_spill_count"]) <= 128, value["name"]
    assert seen == {"mixed": 16, "rows": 54, "blocks": 54, "both": 36}
