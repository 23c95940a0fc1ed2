"""The library's own machine code, as built here: no vector memory instruction reads a scalar register too soon after a vector instruction wrote it.

On this family such a read needs five wait states after the write.  The compiler sees to it for the instructions that it chooses; it does not look into
inline assembly, which has to bring them itself.  No GPU is needed."""
import os
import re
import shutil
import struct
import subprocess

import pytest

WAIT_STATES = 5
OBJDUMP = shutil.which("llvm-objdump", path="/opt/rocm/llvm/bin" + os.pathsep + os.environ.get("PATH", ""))


def code_objects(library):
    """The gfx950 code objects in a library's .hip_fatbin: one bundle for each source file."""
    data = open(library, "rb").read()
    magic, at = b"__CLANG_OFFLOAD_BUNDLE__", 0
    while (at := data.find(magic, at)) >= 0:
        n, p = struct.unpack_from("<Q", data, at + len(magic))[0], at + len(magic) + 8
        if n > 8:  # the word itself, in another section
            at += 1
            continue
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + length]
            p += 24 + length
            if b"gfx950" in name and size:
                yield data[at + offset:at + offset + size]
        at += 1


def scalars(operand):
    """The scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return {f"s{i}" for i in range(int(m[1]), int(m[2]) + 1)}
    return {operand} if re.fullmatch(r"s\d+|vcc_lo|vcc_hi", operand) else {"vcc_lo", "vcc_hi"} if operand == "vcc" else set()


SECOND_RESULT = re.compile(r"v_(add|sub|subrev|addc|subb|subbrev)_co_|v_mad_[ui]64_|v_div_scale_")  # these write a scalar as their second operand


def written(name, operands):
    """The scalar registers that a vector instruction writes."""
    out = scalars(operands[0]) if operands else set()
    return out | scalars(operands[1]) if SECOND_RESULT.match(name) and len(operands) > 1 else out


def too_soon(lines):
    """(function, instruction, wait states) of every vector memory instruction that reads a scalar sooner than it may, and how many instructions there were."""
    found, function, since, memory = [], "", {}, 0
    for line in lines:
        m = re.match(r"[0-9a-f]+ <(.*)>:", line)
        if m:
            if not m[1].startswith("L"):
                function, since = m[1], {}
            continue
        text = line.split("//")[0].strip()
        if not text or ":" in text.split(" ")[0]:
            continue
        name, _, rest = text.partition(" ")
        operands = [o.strip() for part in rest.split(",") for o in part.split(" ") if o.strip()]
        if re.match(r"(global|buffer|flat|scratch)_", name):
            memory += 1
            near = [since[s] for o in operands for s in scalars(o) if s in since]
            if near and min(near) < WAIT_STATES:
                found.append((function, text, min(near)))
        states = int(operands[0], 0) + 1 if name == "s_nop" else 1
        since = {s: n + states for s, n in since.items() if n + states < WAIT_STATES}
        if name.startswith("v_"):
            since.update({s: 0 for s in written(name, operands)})
    return found, memory


def test_the_search_finds_what_it_should():
    head = ["0000000000001000 <kernel>:", "\tv_readlane_b32 s4, v1, s9       // 000000001000: 00000000", "\tv_readlane_b32 s5, v2, s9"]
    load = "\tglobal_load_lds_dwordx4 v3, s[4:5]"
    assert too_soon(head + [load]) == ([("kernel", load.strip(), 0)], 1)
    assert too_soon(head + ["\ts_add_u32 m0, s6, 0x400", "\ts_nop 0", load])[0] == [("kernel", load.strip(), 2)]
    assert too_soon(head + ["\ts_add_u32 m0, s6, 0x400", "\ts_nop 3", load]) == ([], 1)
    assert too_soon(head + ["\ts_nop 4", "\tglobal_load_dword v3, v4, s[4:5] offset:16"]) == ([], 1)
    assert too_soon(head + ["\tglobal_load_dword v3, v4, s[6:7]", "\tglobal_load_dword v3, v[4:5], off"]) == ([], 2)
    assert too_soon(["\tv_cmp_lt_u32_e64 s[0:1], v1, v2", "\tbuffer_load_dword v1, v2, s[0:3], 0 offen"])[0][0][2] == 0
    assert too_soon(["\tv_add_co_u32_e64 v1, s[0:1], v1, v2", "\tglobal_load_dword v3, v4, s[0:1]"])[0][0][2] == 0


@pytest.mark.skipif(OBJDUMP is None, reason="llvm-objdump is not installed")
def test_scalar_addresses_are_waited_for(tmp_path):
    import paper_2511_16138_amd.binding as B
    if not os.path.exists(B.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    found, memory, objects, copies = [], 0, 0, 0
    for i, code in enumerate(code_objects(B.library_path())):
        path = tmp_path / f"{i}.o"
        path.write_bytes(code)
        lines = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], check=True, capture_output=True, text=True).stdout.splitlines()
        f, m = too_soon(lines)
        found, memory, objects = found + f, memory + m, objects + 1
        copies += sum("global_load_lds_dwordx4" in line for line in lines)
    assert objects >= 6 and memory > 1000 and copies > 100  # the search did see the kernels
    assert not found, f"{len(found)} of {memory} read a scalar register too soon, such as {found[:3]}"
