"""Reads across lanes in the built language-model kernels, from their disassembly: a value is read from another lane two instructions after it was
written at the earliest, and the scan's sums over columns keep their eight values in eight registers."""
import os
import re
import struct
import subprocess

import pytest

from paper_2012_15198_amd import cxlm as lm

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{mangled name: [instruction]} of libcxlm.so's kernels that read across lanes."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    data, folder, found = open(lm.LIB_PATH, "rb").read(), tmp_path_factory.mktemp("code"), {}
    for match in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data):
        pos, entry = match.start(), match.start() + 32
        for _ in range(struct.unpack_from("<Q", data, pos + 24)[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            code = data[pos + offset:pos + offset + size]
            if size and b"gfx950" in data[entry + 24:entry + 24 + length]:
                path = folder / f"{pos}.co"
                path.write_bytes(code)
                text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(path)], capture_output=True, text=True, check=True).stdout
                for part in re.split(r"\n(?=<_Z)", text)[1:]:
                    name, body = re.match(r"<(\S+)>:\n(.*)", part, re.S).groups()
                    if "_dpp" in body:
                        found[name] = [line.split("//")[0].strip() for line in body.split("\n") if line.startswith("\t")]
            entry += 24 + length
    return found


def registers(operand):
    """Numbers of the vector registers that an operand names."""
    match = re.fullmatch(r"v(\d+)|v\[(\d+):(\d+)\]", operand.strip("-|"))
    return set() if not match else {int(match[1])} if match[1] else set(range(int(match[2]), int(match[3]) + 1))


def operands(instruction):
    return [o.strip() for o in instruction.split(None, 1)[1].split(",")] if " " in instruction else []


def test_no_value_is_read_across_lanes_too_early(kernels):
    assert len(kernels) > 40
    for name, lines in kernels.items():
        written = []                                         # by each of the last two wait states
        for line in lines:
            op = line.split(None, 1)[0] if line else ""
            if op.endswith("_dpp"):
                source = operands(line)[1].split(" ")[0]
                assert not any(registers(source) & w for w in written[-2:]), (name, line)
            if op == "s_nop":
                written += [set()] * (int(line.split()[1]) + 1)
            else:
                written.append(registers(operands(line)[0]) if op.startswith("v_") and operands(line) else set())


def test_sums_over_columns_keep_their_values_apart(kernels):
    """Groups of fourteen additions: eight in halves of a row of lanes, of four values and then over them of four others."""
    groups = 0
    for name, lines in kernels.items():
        if "select_grad_kernel" not in name:
            continue
        mirrored = [(i, line) for i, line in enumerate(lines) if " row_mirror " in line and line.startswith("v_add_f32_dpp")]
        second = [k for k, (_, line) in enumerate(mirrored) if "bank_mask:0x3" in line]
        for k in second[::4]:
            block = [line for _, line in mirrored[k - 4:k + 4]]
            assert [("bank_mask:0x3" in line) for line in block] == [False] * 4 + [True] * 4, (name, block)
            sums, added = [registers(operands(line)[0]) for line in block[:4]], [registers(operands(line)[1]) for line in block[4:]]
            assert len(set().union(*sums, *added)) == 8, (name, block)
            groups += 1
    assert groups >= 16 * 12                                 # sixteen steps in each of the kernels of three and four states a lane
