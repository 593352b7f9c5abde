"""The loads straight to LDS are written in assembly, which the compiler's own pass for wait states does not look into.  What gfx950
leaves to the program holds in the assembly that the kernels are built to: a wait state between a scalar write of m0 and a load to
LDS, and five between a vector instruction that writes a scalar register of the load's buffer and the load."""
import os
import re
import subprocess

import pytest

from paper_2106_10796_amd import build

SOURCE = os.path.join(build.PKG, "csrc", "mxfp4.hip")


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """(lines of assembly, what the compiler said)"""
    out = str(tmp_path_factory.mktemp("isa") / "mxfp4.s")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-fPIC", "-shared")]
    r = subprocess.run([build.hipcc_path(), *flags, "-I", build.INCLUDE, "--cuda-device-only", "-S", SOURCE, "-o", out],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    with open(out) as fh:
        lines = [line.split(";")[0].strip() for line in fh]
    return [x for x in lines if x and not x.startswith((".", "#")) and not x.endswith(":")], r.stdout


def _scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.fullmatch(r"s(\d+)", operand)
    return {int(m[1])} if m else set()


def _operands(line):
    parts = line.split(None, 1)
    return [o.strip() for o in parts[1].split(",")] if len(parts) > 1 else []


def faults(lines):
    """The loads to LDS that come too soon after a write of what they read: (load, write)."""
    loads, bad = 0, []
    for i, line in enumerate(lines):
        if not (line.startswith("buffer_load") and line.endswith(" lds")):
            continue
        loads += 1
        buffer, states = _scalars(_operands(line)[1]), 0
        assert len(buffer) == 4, line
        for before in reversed(lines[max(i - 5, 0):i]):
            ops = _operands(before)
            written = ops[0] if ops else ""
            if states < 1 and written == "m0":
                bad.append((line, before))
            if states < 5 and before.startswith("v_") and _scalars(written) & buffer:
                bad.append((line, before))
            nop = re.fullmatch(r"s_nop (\d+)", before)
            states += 1 + (int(nop[1]) if nop else 0)
    return loads, bad


def test_wait_states(compiled):
    loads, bad = faults(compiled[0])
    assert loads > 100 and not bad, "%d of %d: %s" % (len(bad), loads, bad[:3])


def test_what_it_would_find():
    load = "buffer_load_dwordx4 v1, s[4:7], 0 offen lds"
    assert faults(["s_mov_b32 m0, s3", load])[1] and not faults(["s_mov_b32 m0, s3", "s_nop 0", load])[1]
    assert faults(["v_readfirstlane_b32 s6, v3", "s_mov_b32 m0, s3", "s_nop 2", load])[1]
    assert not faults(["v_readfirstlane_b32 s6, v3", "s_mov_b32 m0, s3", "s_nop 3", load])[1]
    assert not faults(["v_readfirstlane_b32 s8, v3", "s_nop 0", load])[1]


def test_m0_is_declared_and_nothing_is_said_about_it(compiled):
    """Every piece of assembly that sets m0 says so, and no other instruction of these kernels relies on it."""
    with open(os.path.join(build.PKG, "csrc", "kernels_mxfp4_product.hpp")) as fh:
        pieces = re.findall(r"asm volatile\((.*?)\);", fh.read(), re.S)
    setting = [p for p in pieces if "m0," in p]
    assert setting and all('"m0"' in p.rsplit(":", 1)[1] for p in setting)
    assert "reserved" not in compiled[1]
    uses = [line for line in compiled[0] if re.search(r"\bm0\b", line)]
    assert uses and all(line.startswith("s_mov_b32 m0, s") for line in uses)
