"""The machine code of the token operators' products, as it lies in the library, against three rules that hardware leaves to the program and the compiler
keeps only in its own instructions, not in written-out ones (no GPU needed):
  * a scalar register that a vector instruction wrote is not read by a memory instruction within five wait states;
  * between the setting of m0 and the load into LDS that goes by it nothing else sets m0, and one wait state passes;
  * an accumulation register is read by another instruction than a product 19 wait states (those of the longest product) behind the last one at the earliest."""
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


def loads_off_m0(code):
    """loads into LDS without their own setting of m0 in the three instructions in front"""
    bad = []
    for i, (op, operands) in enumerate(code):
        if op.startswith("buffer_load") and operands.endswith("lds"):
            near = code[max(0, i - 3):i]
            sets = [k for k, (_, o) in enumerate(near) if o.split(",")[0].strip() == "m0"]
            if len(sets) != 1 or sum(waits(*c) for c in near[sets[0] + 1:]) < 1:
                bad.append((near, operands))
    return bad


def early_sums(code):
    """reads of accumulation registers, or copies of them, too close behind the products that wrote them"""
    wrote, now, bad = {}, 0, []
    for op, operands in code:
        regs = [range(int(m[1] or m[2]), int(m[1] or m[3]) + 1) for m in re.finditer(r"\ba(?:(\d+)|\[(\d+):(\d+)\])", operands)]
        if op.startswith("v_mfma"):
            for r in regs[0] if regs and operands.startswith("a") else ():
                wrote[r] = now
        else:
            bad += [(op, operands, r) for s in regs for r in s if r in wrote and now - wrote[r] - 1 < 19]
        now += waits(op, operands)
    return bad


def test_the_scan_sees_what_it_looks_for():
    code = [["v_readfirstlane_b32", "s22, v2"], ["s_mov_b32", "m0, s37"], ["s_nop", "0"], ["buffer_load_dwordx4", "v125, s[20:23], 0 offen lds"]]
    assert early_reads(code) == [("buffer_load_dwordx4", "v125, s[20:23], 0 offen lds", 22, 2)] and not loads_off_m0(code)
    assert not early_reads(code[:1] + [["s_nop", "2"]] + code[1:]) and not early_reads(code[:1] + [["s_mov_b32", "s22, s3"]] + code[1:])
    assert loads_off_m0(code[:2] + code[3:]) and loads_off_m0(code[:1] + code[2:]) and loads_off_m0(code[:2] + code[1:])
    code = [["v_mfma_f32_16x16x32_bf16", "a[0:3], v[14:17], v[62:65], a[0:3]"], ["s_nop", "15"], ["v_accvgpr_read_b32", "v1, a2"]]
    assert early_sums(code) == [("v_accvgpr_read_b32", "v1, a2", 2)] and early_sums(code[:2] + [["ds_write_b128", "v5, a[0:3]"]])
    assert not early_sums(code[:2] + code[1:]) and not early_sums(code[:2] + [["v_accvgpr_read_b32", "v1, a4"]])


def test_descriptors_have_settled_when_loads_read_them(kernels):
    bad = {name: early_reads(code)[:2] for name, code in kernels.items()}
    bad = {k: v for k, v in bad.items() if v}
    assert not bad, (len(bad), list(bad.items())[:3])


def test_loads_into_lds_go_by_their_own_m0(kernels):
    assert all(any(o.endswith("lds") for _, o in code) for name, code in kernels.items())
    bad = {name: loads_off_m0(code)[:2] for name, code in kernels.items()}
    assert not any(bad.values()), [(k, v) for k, v in bad.items() if v][:3]


def test_sums_are_read_when_they_are_there(kernels):
    large = {name: code for name, code in kernels.items() if "tg_big_k" in name}
    assert len(large) == 10 and all(any(op.startswith("v_mfma") and o.startswith("a[") for op, o in code) for code in large.values())
    bad = {name: early_sums(code)[:2] for name, code in large.items()}
    assert not any(bad.values()), [(k, v) for k, v in bad.items() if v][:3]
