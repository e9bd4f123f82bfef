"""The machine code of the built library: what hand-written assembly statements have to see to by themselves, because the compiler does
not look into them."""
import os
import re
import struct
import subprocess

import pytest

from paper_2104_11487_amd import skipconv as S
from paper_2104_11487_amd.build import ARCH, hipcc

OBJDUMP = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(hipcc()))), "llvm", "bin", "llvm-objdump")


def code_objects(path):
    """The device code objects of a library, from its offload bundles: 24 bytes of magic, a count, and for each entry offset, size and name."""
    data = open(path, "rb").read()
    at = data.find(b"__CLANG_OFFLOAD_BUNDLE__")
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        entry = at + 32
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            if ARCH.encode() in data[entry + 24:entry + 24 + length]:
                yield data[at + offset:at + offset + size]
            entry += 24 + length
        at = data.find(b"__CLANG_OFFLOAD_BUNDLE__", entry)


SCALAR = re.compile(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b|\b(vcc)\b")
INSTRUCTION = re.compile(r"^\t(\w+) ?([^/]*)")
MEMORY = ("global_", "buffer_", "flat_", "scratch_")


def scalars(text):
    """Numbers of the scalar registers that an operand list names."""
    for first, last, one, vcc in SCALAR.findall(text):
        yield from range(int(first), int(last) + 1) if first else [int(one)] if one else [-1, -2]


def least_wait_states(listing):
    """For each kind of memory load with a scalar register that a vector instruction wrote: the least wait states between the two (each
    instruction is one, s_nop n is n + 1), in the order of the listing. And how many such loads there were."""
    least, loads, written, now = {}, 0, {}, 0
    for line in listing:
        if line.endswith(">:"):
            written = {}
            continue
        m = INSTRUCTION.match(line)
        if not m:
            continue
        op, args = m.groups()
        if op == "s_nop":
            now += int(args, 0) + 1
            continue
        if op.startswith(MEMORY):
            since = [now - written[r] - 1 for r in scalars(args) if r in written]
            if since:
                loads += 1
                least[op] = min([least.get(op, 1 << 30)] + since)
        elif op.startswith("v_"):
            operands = args.split(",")
            to = "vcc" if op.startswith("v_cmp") and op.endswith("_e32") else operands[0]
            if "_co_" in op or op.startswith(("v_mad_u64", "v_mad_i64", "v_div_scale")):
                to += "," + operands[1]
            for r in scalars(to):
                written[r] = now
        elif op.startswith("s_") and not op.startswith(("s_cmp", "s_bitcmp", "s_cbranch", "s_branch", "s_wait", "s_barrier", "s_setprio")):
            for r in scalars(args.split(",")[0]):
                written.pop(r, None)
        now += 1
    return least, loads


def test_the_count_of_wait_states():
    text = ["0 <kernel>:", "\tv_readlane_b32 s5, v1, 3  // x", "\ts_mov_b32 m0, s9 // x", "\ts_nop 1 // x", "\tglobal_load_lds_dwordx4 v0, s[4:5] // x"]
    assert least_wait_states(text) == ({"global_load_lds_dwordx4": 3}, 1)
    assert least_wait_states(text[:2] + ["\ts_mov_b32 s5, s7 // x"] + text[3:]) == ({}, 0)
    assert least_wait_states(["\tv_cmp_eq_u32_e32 v1, v2 // x", "\tglobal_load_dword v0, v1, vcc // x"]) == ({"global_load_dword": 0}, 1)


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs llvm-objdump of ROCm")
def test_scalar_addresses_have_settled(tmp_path):
    """A memory instruction may read a scalar register from the fifth wait state after a vector instruction wrote it (v_readlane: the
    bases of the copies into LDS)."""
    seen = 0
    for i, code in enumerate(code_objects(S.LIB_PATH)):
        if b"attend" not in code:  # the units with such statements
            continue
        path = tmp_path / f"{i}.co"
        path.write_bytes(code)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
        least, loads = least_wait_states(text.splitlines())
        assert all(n >= 5 for n in least.values()), least
        seen += loads
    assert seen > 100
