"""Checks on the sources and the generated gfx950 code of the feed-forward kernels (no GPU needed).

A load into LDS is written as an instruction, with its resource in scalar registers and m0 set in front of it.  The compiler has to be told of
m0, and it must not have put vector registers where the text expects scalar ones."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2011_05630_amd", "csrc")


def test_assembly_names_what_it_writes():
    seen = 0
    for f in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, f)) as s:
            for m in re.finditer(r"\basm\b[^;]*?\(((?:\"(?:[^\"\\]|\\.)*\"|[^;\"])*)\);", s.read()):
                if re.search(r"s_mov_b32 m0", m.group(1)):
                    seen += 1
                    assert re.search(r"\"m0\"", m.group(1).rsplit(":", 1)[1]), (f, m.group(0))
    assert seen >= 6


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("ff") / "ffn.s")
    r = subprocess.run(["hipcc", "-O3", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", "-S", "--cuda-device-only", "-Xclang", "-target-feature", "-Xclang",
                        "-packed-fp32-ops", "-Wno-unused-command-line-argument", "-o", out, os.path.join(CSRC, "dlf_ffn.hip")],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    with open(out) as f:
        return f.read()


def test_loads_into_lds_have_scalar_resources(asm):
    loads = re.findall(r"^\s*buffer_load_dwordx4 (.*\blds)\b", asm, flags=re.M)
    assert len(loads) > 100
    for ops in loads:
        assert re.match(r"^v\d+, s\[\d+:\d+\], 0 offen lds$", ops.strip()), ops


def test_no_kernel_spills_to_scratch(asm):
    sizes = re.findall(r"^\s*\.amdhsa_kernel\s+(\S+).*?\.amdhsa_private_segment_fixed_size\s+(\d+)", asm, flags=re.M | re.S)
    assert len(sizes) > 30
    assert {n: b for n, b in sizes if int(b) > 0} == {}
