"""The built library's machine code keeps the wait states that the hardware asks of
the program.  The compiler sees to them between its own instructions and not
inside or around inline assembly, so the whole library is disassembled and read
in the order of its text (no GPU needed)."""
import concurrent.futures as cf
import os
import re
import struct
import subprocess

import pytest

import paper_2212_14052_amd as h3

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
BUNDLE = b"__CLANG_OFFLOAD_BUNDLE__"
# of a matrix instruction: states before its summand's registers may be written, before its result may be read or written
MATRIX = {"v_mfma_f32_16x16x32_f16": (3, 8), "v_mfma_f32_16x16x32_bf16": (3, 8), "v_mfma_f32_32x32x16_f16": (7, 12),
          "v_mfma_f32_32x32x16_bf16": (7, 12), "v_mfma_f32_16x16x4_f32": (7, 10)}
REG = re.compile(r"\b([vsa])(\d+)\b|\b([vsa])\[(\d+):(\d+)\]|\b(m0|vcc)\b")


def code_objects(path):
    """The gfx950 code objects in a shared library."""
    data, at = open(path, "rb").read(), 0
    while (at := data.find(BUNDLE, at)) >= 0:
        start, at = at, at + len(BUNDLE)
        count, = struct.unpack_from("<Q", data, at)
        p = at + 8
        for _ in range(count if count < 16 else 0):
            off, size, n = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + n]
            p += 24 + n
            if b"gfx950" in name:
                yield data[start + off:start + off + size]


def registers(operand):
    found = set()
    for kind, n, kinds, lo, hi, name in REG.findall(operand):
        if kind:
            found.add(kind + n)
        elif kinds:
            found.update(f"{kinds}{i}" for i in range(int(lo), int(hi) + 1))
        else:
            found.add(name)
    return found


class Instruction:
    def __init__(self, text):
        self.text = text
        self.name, _, rest = text.partition(" ")
        ops = [registers(o) for o in re.split(r",(?![^\[]*\])", rest)] if rest else []
        self.states = int(rest, 0) + 1 if self.name == "s_nop" else 1
        self.matrix = self.name.startswith("v_mfma")
        self.vector = self.name.startswith("v_") and not self.matrix
        self.memory = self.name.startswith(("global_", "buffer_", "scratch_", "flat_"))
        into_lds = self.memory and "lds" in self.name
        keeps = into_lds or (self.memory and "store" in self.name) or self.name.startswith(("ds_write", "s_cmp", "s_cbranch", "s_waitcnt"))
        self.into_lds = into_lds
        self.writes = ops[0] if ops and not keeps else set()
        self.reads = set().union(set(), *(ops if keeps else ops[1:]))
        self.summand = ops[3] if self.matrix else set()
        if self.name.startswith(("v_fmac", "v_fma_mixhi")):
            self.reads |= self.writes


def missing(before, states, now):
    """What `now` still lacks, `states` wait states behind `before`."""
    if now.into_lds and "m0" in before.writes and states < 1:
        return "a write of m0, then a copy into LDS"
    if now.memory and before.vector and states < 5 and any(r[0] == "s" or r == "vcc" for r in before.writes & now.reads):
        return "a scalar register written by a vector instruction, then an address in it"
    if now.matrix and before.vector and states < 2 and before.writes & now.reads:
        return "a vector instruction's result into a matrix instruction"
    if before.matrix and (now.vector or now.memory or now.name.startswith("ds_")):
        summand, result = MATRIX[before.name]
        if states < summand and before.summand & now.writes:
            return "a matrix instruction's summand, overwritten"
        if states < result and before.writes & (now.reads | now.writes):
            return "a matrix instruction's result, read or overwritten"
    return None


def faults(listing):
    found, window = [], []
    for line in listing.splitlines():
        if line.endswith(">:"):
            kernel, window = line.split("<")[1][:-2], []
            continue
        text = line.split("//")[0].strip()
        if not line.startswith("\t") or not text:
            continue
        now, states = Instruction(text), 0
        for before in reversed(window):
            what = missing(before, states, now)
            if what:
                found.append(f"{kernel}: {what}: {before.text}; {now.text}")
            states += before.states
            if states > 20:
                break
        window = [] if now.name in ("s_branch", "s_endpgm", "s_setpc_b64") else (window + [now])[-20:]
    return found


def disassemble_and_read(args):
    path, code = args
    with open(path, "wb") as f:
        f.write(code)
    r = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], capture_output=True, text=True, check=True)
    return len(r.stdout), faults(r.stdout)


@pytest.mark.parametrize("text,count", [
    ("s_mov_b32 m0, s4\n\tglobal_load_lds_dwordx4 v1, s[2:3]", 1),
    ("s_mov_b32 m0, s4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 v1, s[2:3]", 0),
    ("v_readfirstlane_b32 s3, v0\n\ts_nop 3\n\tglobal_load_dword v1, v2, s[2:3]", 1),
    ("v_readfirstlane_b32 s3, v0\n\ts_nop 4\n\tglobal_load_dword v1, v2, s[2:3]", 0),
    ("v_add_f32_e32 v1, v2, v3\n\tv_mfma_f32_16x16x32_f16 v[4:7], v[0:3], v[8:11], 0", 1),
    ("v_add_f32_e32 v1, v2, v3\n\ts_nop 1\n\tv_mfma_f32_16x16x32_f16 v[4:7], v[0:3], v[8:11], 0", 0),
    ("v_mfma_f32_16x16x32_f16 v[4:7], v[0:3], v[8:11], v[12:15]\n\ts_nop 1\n\tv_fma_mixlo_f16 v14, v20, v21, 0", 1),
    ("v_mfma_f32_16x16x32_f16 v[4:7], v[0:3], v[8:11], v[12:15]\n\ts_nop 2\n\tv_fma_mixlo_f16 v14, v20, v21, 0", 0),
    ("v_mfma_f32_16x16x32_f16 v[4:7], v[0:3], v[8:11], 0\n\ts_nop 6\n\tv_add_f32_e32 v20, v20, v4", 1),
    ("v_mfma_f32_16x16x32_f16 v[4:7], v[0:3], v[8:11], 0\n\ts_nop 7\n\tv_add_f32_e32 v20, v20, v4", 0),
    ("v_mfma_f32_16x16x32_f16 v[4:7], v[0:3], v[8:11], 0\n\ts_branch 9\n\tv_add_f32_e32 v20, v20, v4", 0),
])
def test_the_reader(text, count):
    assert len(faults("0 <k>:\n\t" + text + "\n")) == count


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs llvm-objdump")
def test_library(tmp_path):
    h3.lib()
    objects = list(code_objects(h3.LIB_PATH))
    assert len(objects) >= 10
    with cf.ProcessPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        results = list(pool.map(disassemble_and_read, [(str(tmp_path / f"{i}.elf"), code) for i, code in enumerate(objects)]))
    assert sum(size for size, _ in results) > 1 << 20
    found = [f for _, fs in results for f in fs]
    assert not found, "\n".join(found[:20]) + f"\n{len(found)} in all"
