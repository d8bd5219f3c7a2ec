"""Registers of the built language-model kernels, from the metadata that the compiler leaves in the library: none keeps
registers in scratch memory, which the runtime would allocate on a first launch, and the ones that hold a row leave a CU
the workgroups they are meant for."""
import os
import re
import struct
import subprocess

import pytest

from paper_2012_15198_amd import cxlm as lm

READELF = "/opt/rocm/llvm/bin/llvm-readelf"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """[(mangled name, registers, scratch bytes)] of libcxlm.so."""
    if not os.path.exists(READELF):
        pytest.skip("no llvm-readelf")
    data, folder, found = open(lm.LIB_PATH, "rb").read(), tmp_path_factory.mktemp("code"), []
    for match in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data):
        pos, entry = match.start(), match.start() + 32
        for _ in range(struct.unpack_from("<Q", data, pos + 24)[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            if size and b"gfx950" in data[entry + 24:entry + 24 + length]:
                path = folder / f"{pos}.co"
                path.write_bytes(data[pos + offset:pos + offset + size])
                notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
                for block in re.split(r"\n\s*- \.agpr_count", notes)[1:]:
                    number = {key: int(value) for key, value in re.findall(r"\.(\w+):\s+(\d+)\s*$", block, re.M)}
                    found.append((re.search(r"\.name:\s+(_Z\S+)", block).group(1), number["vgpr_count"], number["private_segment_fixed_size"]))
            entry += 24 + length
    return found


def test_no_kernel_keeps_registers_in_scratch(kernels):
    assert len(kernels) > 60 and not [k for k in kernels if k[2]]


def test_rows_in_registers_leave_room_for_a_second_workgroup(kernels):
    rows = [(name, vgpr) for name, vgpr, _ in kernels if "row_kernel" in name]
    assert len(rows) >= 36
    for name, vgpr in rows:
        assert vgpr <= (128 if "Li16E" in name else 64), name


def test_recurrence_keeps_two_wavefronts_a_simd(kernels):
    scans = [(name, vgpr) for name, vgpr, _ in kernels if "scan_kernel" in name or "scan_grad_kernel" in name]
    assert len(scans) >= 36 and all(vgpr <= 256 for _, vgpr in scans)


def test_scores_keep_eight_wavefronts_a_simd(kernels):
    scores = [(name, vgpr) for name, vgpr, _ in kernels if "scores_kernel" in name]
    assert len(scores) >= 18 and all(vgpr <= 64 for _, vgpr in scores)
