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


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    """The instructions of each device image in the built library."""
    objdump = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"
    if not os.path.exists(objdump):
        pytest.skip("no llvm-objdump")
    if not os.path.exists(dptq.library_path()):
        B.build()
    path = tmp_path_factory.mktemp("images")
    lib = shutil.copy(dptq.library_path(), path)
    subprocess.run([objdump, "--offloading", lib], cwd=path, check=True, stdout=subprocess.DEVNULL)
    images = []
    for image in sorted(glob.glob(str(path / f"*{B.ARCH}*"))):
        out = subprocess.run([objdump, "-d", "--no-show-raw-insn", "--no-leading-addr", image], check=True,
                             capture_output=True, text=True).stdout
        images.append([line.split("//")[0].strip() for line in out.splitlines()])
    return images


def test_built_library_waits_for_m0(listings):
    loads = 0
    for listing in listings:
        n, bad = missing_waits(listing)
        loads += n
        assert not bad, (len(bad), bad[:3])
    assert loads > 0


def scalars(operand):
    """The scalar registers that an operand names."""
    m = re.match(r"s(?:(\d+)|\[(\d+):(\d+)\])$", operand)
    return set() if not m else {int(m[1])} if m[1] else set(range(int(m[2]), int(m[3]) + 1))


def late_bases(listing):
    """Direct loads less than five wait states behind a vector instruction's write of their scalar base."""
    window, bad = [], []
    for i in listing:
        parts = i.replace(",", " ").split()
        if not parts or i.endswith(":"):
            continue
        if "_load_lds_" in parts[0]:
            base, states = set().union(*map(scalars, parts[1:])), 0
            for p in reversed(window):
                if p[0].startswith("v_") and len(p) > 1 and scalars(p[1]) & base:
                    bad.append((p[0], i))
                states += int(p[1], 0) + 1 if p[0] == "s_nop" else 1
                if states >= 5:
                    break
        window = (window + [parts])[-5:]
    return bad


def test_built_library_waits_for_scalar_bases(listings):
    # The other wait that the compiler leaves out of an asm statement: a scalar register that a vector instruction
    # writes (a lane that is read) is a load's base five wait states later at the earliest.
    load = "global_load_lds_dwordx4 v1, s[2:3]"
    write = "v_readlane_b32 s3, v9, 1"
    assert late_bases([write, "s_mov_b32 m0, s4", "s_nop 0", load]) == [("v_readlane_b32", load)]
    assert late_bases([write, "s_mov_b32 m0, s4", "s_nop 3", load]) == []
    for listing in listings:
        bad = late_bases(listing)
        assert not bad, (len(bad), bad[:3])
