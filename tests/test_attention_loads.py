"""Attention's loads straight to LDS: the wait states that gfx950 leaves to the program hold in the assembly that the kernels are built to, and
kernels hold what they keep in registers."""
import os
import re
import subprocess

import pytest

from paper_2106_10796_amd import build
from test_loads_to_lds import faults


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("isa") / "attention.s")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-fPIC", "-shared")]
    r = subprocess.run([build.hipcc_path(), *flags, "-I", build.INCLUDE, "--cuda-device-only", "-S", os.path.join(build.PKG, "csrc", "attention.hip"), "-o", out],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    with open(out) as fh:
        return fh.read()


def test_wait_states(compiled):
    lines = [line.split(";")[0].strip() for line in compiled.splitlines()]
    lines = [x for x in lines if x and not x.startswith((".", "#")) and not x.endswith(":")]
    loads, bad = faults(lines)
    assert loads > 50 and not bad, "%d of %d: %s" % (len(bad), loads, bad[:3])
    uses = [line for line in lines if re.search(r"\bm0\b", line)]
    assert uses and all(line.startswith("s_mov_b32 m0, s") for line in uses)


def test_nothing_of_bf16_is_kept_in_scratch(compiled):
    """A reload in a loop would wait for every load to LDS that is under way."""
    sizes = dict(re.findall(r"\.amdhsa_kernel (_ZN\S+)\n.*?\.amdhsa_private_segment_fixed_size (\d+)", compiled, re.S))
    mine = {k: int(v) for k, v in sizes.items() if "k_attention" in k and "ILi1E" in k}
    assert len(mine) == 8 and not any(mine.values()), mine
