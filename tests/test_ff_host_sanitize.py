"""The host side of the feed-forward operators under AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU.

tests/ff_host_driver.cpp is compiled together with csrc/dlf_ffn.cpp, host code instrumented, the launchers replaced by stand-ins that check each
launch against what its kernels assume: operands in whole lines where tiles are loaded directly, workgroups and threads within a launch's
limit, everything kept in the workspace inside it and apart, sums and gradients asked for and no others.  Random calls of the four
operations: sizes from one to the limits and around them, strides, alignments, subsets of the gradients, kernels and splits by the rule and forced."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("ffsan") / "ff_host_driver")
    host = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
            "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    cmd = (["hipcc", "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-x", "hip"] + host +
           ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument", "-o", exe,
            os.path.join(ROOT, "tests", "ff_host_driver.cpp"), os.path.join(ROOT, "paper_2011_05630_amd", "csrc", "dlf_ffn.cpp")])
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    return exe


def test_driver_replaces_every_launcher():
    def names(*path):
        with open(os.path.join(ROOT, *path)) as f:
            return set(re.findall(r"int (dlf_ff_(?:start|kernels)_\w+)\(", f.read()))
    assert names("paper_2011_05630_amd", "csrc", "dlf_ffn.h") == names("tests", "ff_host_driver.cpp")


@pytest.mark.parametrize("seed", range(1, 5))
def test_random_calls(driver, seed):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:halt_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([driver, str(seed), "60000"], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, env=env, timeout=600)
    assert r.returncode == 0, "status %d\n%s\n%s" % (r.returncode, r.stdout[-2000:], r.stderr[-6000:])
    assert "runtime error" not in r.stderr and "Sanitizer" not in r.stderr, r.stderr[-6000:]
    m = re.match(r"calls 60000 ok (\d+) invalid (\d+) unsupported (\d+) split (\d+) seen ([\d ]+)$", r.stdout.strip())
    assert m and int(m.group(1)) > 50000 and int(m.group(3)) > 0 and int(m.group(4)) > 1000
    assert all(int(n) > 100 for n in m.group(5).split())          # every shape, both few-rows kernels, the pass before the products


def test_kernels_are_set_up_on_every_device(driver):
    """Once each, on the calls' first use of it; a device that fails stays refused, the others run."""
    r = subprocess.run([driver, "devices"], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr[-3000:]
    assert r.stdout.strip() == "setups" + " 1" * 8
