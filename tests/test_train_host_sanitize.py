"""The host side of the cross entropy and of the optimizer under AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU.

tests/train_host_driver.cpp is compiled together with csrc/dlf_ce.cpp, csrc/dlf_ffn.cpp and csrc/dlf_opt.cpp, host code instrumented, the launchers replaced by
stand-ins that check each launch against what its kernels assume: operands in whole lines where tiles are loaded directly, workgroups and threads
within a launch's limit, everything kept in the workspace inside it and apart, every row of every piece once, one launch that counts a step."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2011_05630_amd", "csrc")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("trainsan") / "train_host_driver")
    host = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
            "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    cmd = (["hipcc", "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-x", "hip"] + host +
           ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument", "-o", exe,
            os.path.join(ROOT, "tests", "train_host_driver.cpp")] + [os.path.join(CSRC, f) for f in ("dlf_ce.cpp", "dlf_ffn.cpp", "dlf_opt.cpp")])
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    return exe


def test_driver_replaces_every_launcher():
    def names(*path):
        with open(os.path.join(ROOT, *path)) as f:
            return set(re.findall(r"int (dlf_(?:ff|ce|opt)_(?:start|kernels)_\w+)\(", f.read()))
    want = set()
    for h in ("dlf_ffn.h", "dlf_ce.h", "dlf_opt.h"):
        want |= names("paper_2011_05630_amd", "csrc", h)
    assert want == names("tests", "train_host_driver.cpp") and len(want) > 10


@pytest.mark.parametrize("seed", range(1, 4))
def test_random_calls(driver, seed):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:halt_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([driver, str(seed), "15000"], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, env=env, timeout=600)
    assert r.returncode == 0, "status %d\n%s\n%s" % (r.returncode, r.stdout[-2000:], r.stderr[-6000:])
    assert "runtime error" not in r.stderr and "Sanitizer" not in r.stderr, r.stderr[-6000:]
    m = re.match(r"calls 15000 ok (\d+) invalid (\d+) unsupported (\d+) seen (.*)$", r.stdout.strip())
    assert m and int(m.group(1)) > 10000 and int(m.group(3)) > 0
    seen = dict((k, int(v)) for k, v in re.findall(r"\[([^\]]+)\] (\d+)", m.group(4)))
    shapes = (0, 1, 2, 3, 4)
    want = {"mode%d shape%d" % (a, s) for a in (0, 1, 2, 3) for s in shapes} | {"back shape%d" % s for s in shapes}
    want |= {"pack", "few", "few lines", "join", "dz", "dz with lse", "dz few", "dz sums", "dz few with lse", "dz sums with lse", "dz of logits", "unit", "split", "norm", "step", "step small"}
    assert want == set(seen) and all(n >= 10 for n in seen.values()), seen
