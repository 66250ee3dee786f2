"""The machine code of the token operators' products, as it lies in the library, against what hardware leaves to the program and the compiler
keeps only in its own instructions, not in written-out ones (no GPU needed):
  * a scalar register that a vector instruction wrote is not read by a memory instruction within five wait states."""
import os
import re
import shutil
import struct
import subprocess

import pytest

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(data):
    """the gfx950 code objects of the bundles in a shared library"""
    at = data.find(MAGIC)
    while at >= 0:
        n, = struct.unpack_from("<Q", data, at + 24)
        p = at + 32
        for _ in range(n):
            off, size, length = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + length].decode()
            p += 24 + length
            if "gfx950" in name and size:
                yield data[at + off:at + off + size]
        at = data.find(MAGIC, at + 1)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel: its instructions (name, operands)} of the products that load into LDS"""
    import paper_2110_02781_amd as P
    tool = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"
    if not os.path.exists(tool):
        pytest.skip("no llvm-objdump")
    found = {}
    with open(P.binding._LIB_PATH, "rb") as f:
        data = f.read()
    for i, code in enumerate(code_objects(data)):
        if b"tg_gemm_k" not in code and b"tg_big_k" not in code:
            continue
        path = tmp_path_factory.mktemp("code") / f"{i}.o"
        path.write_bytes(code)
        text = subprocess.run([tool, "-d", "--no-show-raw-insn", str(path)], check=True, stdout=subprocess.PIPE, text=True).stdout
        for name, body in re.findall(r"^[0-9a-f]+ <(\S+)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", text, re.S | re.M):
            if "tg_gemm_k" in name or "tg_big_k" in name:
                lines = [line.split("//")[0].strip() for line in body.splitlines()]
                found[name] = [(line.split(None, 1) + [""])[:2] for line in lines if line]
    assert len(found) >= 50, len(found)
    return found


def scalars(operand):
    m = re.fullmatch(r"s(\d+)|s\[(\d+):(\d+)\]", operand.strip())
    if not m:
        return set()
    return {int(m[1])} if m[1] else set(range(int(m[2]), int(m[3]) + 1))


def waits(op, operands):
    return int(operands, 0) + 1 if op == "s_nop" else 1


def early_reads(code):
    """memory instructions that read a scalar register fewer than five wait states behind the vector instruction that wrote it"""
    wrote, now, bad = {}, 0, []
    for op, operands in code:
        parts = operands.split(",")
        if op.startswith(("buffer_", "global_")):
            # of a register range only the last operands' modifiers follow without a comma
            for part in parts:
                for r in scalars(part.split()[0] if part.split() else ""):
                    if r in wrote and now - wrote[r] - 1 < 5:
                        bad.append((op, operands, r, now - wrote[r] - 1))
        elif op.startswith("v_"):
            for r in scalars(parts[0]):
                wrote[r] = now
        elif op.startswith("s_") and parts[0]:
            for r in scalars(parts[0]):
                wrote.pop(r, None)
        now += waits(op, operands)
    return bad


def test_the_scan_sees_what_it_looks_for():
    code = [["v_readfirstlane_b32", "s22, v2"], ["s_mov_b32", "m0, s37"], ["s_nop", "0"], ["buffer_load_dwordx4", "v125, s[20:23], 0 offen lds"]]
    assert early_reads(code) == [("buffer_load_dwordx4", "v125, s[20:23], 0 offen lds", 22, 2)]
    assert not early_reads(code[:1] + [["s_nop", "2"]] + code[1:]) and not early_reads(code[:1] + [["s_mov_b32", "s22, s3"]] + code[1:])


def test_descriptors_have_settled_when_loads_read_them(kernels):
    bad = {name: early_reads(code)[:2] for name, code in kernels.items()}
    bad = {k: v for k, v in bad.items() if v}
    assert not bad, (len(bad), list(bad.items())[:3])
