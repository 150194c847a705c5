"""Checks on the generated gfx950 code of the cross entropy's and the optimizer's kernels (no GPU needed): what test_ff_build.py looks for in the
feed-forward kernels, and that no load of the epilogue has made its way into the wait of a main loop."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2011_05630_amd", "csrc")


@pytest.fixture(scope="module", params=["dlf_ce.hip", "dlf_opt.hip"])
def asm(request, tmp_path_factory):
    out = str(tmp_path_factory.mktemp("train") / (request.param + ".s"))
    r = subprocess.run(["hipcc", "-O3", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", "-S", "--cuda-device-only", "-Xclang", "-target-feature", "-Xclang",
                        "-packed-fp32-ops", "-Wno-unused-command-line-argument", "-o", out, os.path.join(CSRC, request.param)],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    with open(out) as f:
        return request.param, f.read()


def test_generated_code(asm):
    name, text = asm
    sizes = re.findall(r"^\s*\.amdhsa_kernel\s+(\S+).*?\.amdhsa_private_segment_fixed_size\s+(\d+)", text, flags=re.M | re.S)
    assert len(sizes) > (50 if name == "dlf_ce.hip" else 3)
    assert {n: b for n, b in sizes if int(b) > 0} == {}                     # nothing spills to scratch
    loads = re.findall(r"^\s*buffer_load_dwordx4 (.*\blds)\b", text, flags=re.M)
    assert len(loads) > 100 or name == "dlf_opt.hip"
    for ops in loads:
        assert re.match(r"^v\d+, s\[\d+:\d+\], 0 offen lds$", ops.strip()), ops
    assert not re.search(r"v_pk_(add|mul|fma)_f32", text)


def test_main_loops_wait_once_a_stage_for_loads(asm):
    """In the loops over whole stages of the tiles loaded directly, the only waits for loads are the one in front of the barrier."""
    name, text = asm
    if name != "dlf_ce.hip":
        return
    seen = 0
    for m in re.finditer(r"^(_Z\w*k_ce_(?:back|tile)\S*ELb1E\S*):.*?^\.Lfunc_end\d+:", text, flags=re.M | re.S):
        lines = m.group(0).split("\n")
        at = {q.group(1): i for i, q in enumerate(re.match(r"^(\.LBB\w+):", l) for l in lines) if q}
        for i, l in enumerate(lines):
            q = re.search(r"s_c?branch\w*\s+(\.LBB\w+)", l)
            if not q or at.get(q.group(1), i) >= i:
                continue
            body = lines[at[q.group(1)]:i + 1]
            mma = sum("v_mfma" in b for b in body)
            if mma >= 16 and any("s_barrier" in b for b in body) and len(body) < 1000:
                waits = [b for b in body if "s_waitcnt" in b and "vmcnt" in b]
                assert len(waits) <= 1, (m.group(1), waits)
                seen += 1
    assert seen >= 20
