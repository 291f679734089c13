"""Direct loads into LDS take their LDS base from M0, and a scalar write of M0 needs one wait state before such a
load.  The compiler keeps it in its own code and inserts nothing inside an asm statement: checked in the sources'
asm statements and in the instructions of the built library."""

import glob
import os
import re
import shutil
import subprocess

import pytest

import paper_2606_12487_amd as dptq
from paper_2606_12487_amd import build as B


def instructions(asm):
    """The instructions of an asm statement's string literals."""
    text = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', asm.split(":")[0]))
    return [i.strip() for i in text.replace("\\t", " ").split("\\n") if i.strip()]


def missing_waits(listing):
    """Direct loads that follow a write of M0 without another instruction between."""
    before, bad, loads = "", [], 0
    for i in listing:
        if "_load_lds_" in i:
            loads += 1
            if re.match(r"s_\w+\s+m0\b", before):
                bad.append((before, i))
        before = i
    return loads, bad


def test_the_check_itself():
    load = "global_load_lds_dwordx4 v1, s[2:3]"
    assert missing_waits(["s_mov_b32 m0, s4", load]) == (1, [("s_mov_b32 m0, s4", load)])
    assert missing_waits(["s_add_u32 m0, s4, 16", "s_nop 0", load, load]) == (2, [])


def test_sources_wait_for_m0():
    loads = 0
    for path in sorted(glob.glob(os.path.join(B.CSRC, "*"))):
        code = re.sub(r"//[^\n]*", "", open(path).read())
        for asm in re.findall(r"\basm\b[^;]*;", code):
            n, bad = missing_waits(instructions(asm))
            loads += n
            assert not bad, (os.path.basename(path), bad)
    assert loads > 0


def test_built_library_waits_for_m0(tmp_path):
    objdump = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"
    if not os.path.exists(objdump):
        pytest.skip("no llvm-objdump")
    if not os.path.exists(dptq.library_path()):
        B.build()
    lib = shutil.copy(dptq.library_path(), tmp_path)
    subprocess.run([objdump, "--offloading", lib], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    loads = 0
    for image in sorted(glob.glob(str(tmp_path / f"*{B.ARCH}*"))):
        out = subprocess.run([objdump, "-d", "--no-show-raw-insn", "--no-leading-addr", image], check=True,
                             capture_output=True, text=True).stdout
        n, bad = missing_waits([line.split("//")[0].strip() for line in out.splitlines()])
        loads += n
        assert not bad, (len(bad), bad[:3])
    assert loads > 0
