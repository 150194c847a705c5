"""Compile libdlf.so (HIP kernels + host planner) for gfx950 with hipcc, in-tree."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdlf.so")
SOURCES = ["dlf_kernels.hip", "dlf_host.cpp", "dlf_ffn.hip", "dlf_ffn.cpp"]
HEADERS = ["dlf_internal.h", "dlf_ffn.h", os.path.join("..", "..", "include", "dlf.h"),
           os.path.join("..", "..", "include", "dlf_debug.h")]


# The feed-forward operators on PyTorch's tensors; links against libdlf.so beside it and the libraries of the PyTorch it is built with.
TORCH_SOURCE = "dlf_torch.cpp"
TORCH_LIB = os.path.join(HERE, "_dlf_torch.so")


def _older(target, sources):
    t = os.path.getmtime(target)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in sources)


def needs_build():
    return not os.path.exists(LIB) or _older(LIB, SOURCES + HEADERS)


def _built_with():
    import torch
    return "built with PyTorch " + torch.__version__


def needs_build_torch():
    """Missing, older than its sources, or built with another PyTorch than the one installed (it names its own)."""
    if not os.path.exists(TORCH_LIB) or _older(TORCH_LIB, [TORCH_SOURCE, os.path.join("..", "..", "include", "dlf.h")]):
        return True
    with open(TORCH_LIB, "rb") as f:
        return _built_with().encode() not in f.read()


def _run(cmd, target, tmp):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("%s failed:\n%s" % (cmd[0], out))
    if out.strip():
        print(out)
    os.replace(tmp, target)


def build_torch():
    import sysconfig
    import torch
    from torch.utils import cpp_extension as ext
    tmp = TORCH_LIB + ".tmp.%d" % os.getpid()
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           '-DDLF_BUILT_WITH="%s"' % _built_with(), "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
    cmd += ["-I" + p for p in ext.include_paths() + [sysconfig.get_paths()["include"]]]
    cmd += ["-o", tmp, os.path.join(CSRC, TORCH_SOURCE), "-L" + HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"]
    for p in ext.library_paths():
        cmd += ["-L" + p, "-Wl,-rpath," + p]
    _run(cmd + ["-lc10", "-ltorch_cpu", "-ltorch_python"], TORCH_LIB, tmp)


def build(force=True, verbose=False, library_only=False):
    """libdlf.so, and the module on PyTorch's tensors unless `library_only`: a program of the C calls needs hipcc alone."""
    if force or needs_build():
        tmp = LIB + ".tmp.%d" % os.getpid()
        cmd = ["hipcc", "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared", "-Wl,-soname," + os.path.basename(LIB),
               "-x", "hip",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-Wno-unused-command-line-argument",
               "-Wno-inline-asm",               # (statements that write m0 name it as clobbered, which the compiler remarks on)
               "-o", tmp] + [os.path.join(CSRC, s) for s in SOURCES]
        if verbose:
            cmd.insert(1, "-save-temps=obj")
        _run(cmd, LIB, tmp)
    if library_only:
        return LIB
    try:
        import torch  # noqa: F401
    except ImportError:
        print("PyTorch is not installed: built without the operators on its tensors (%s)" % os.path.basename(TORCH_LIB))
        return LIB
    if force or needs_build_torch():
        build_torch()
    return LIB


if __name__ == "__main__":
    import argparse
    parser = argparse.ArgumentParser(description=__doc__)
    parser.add_argument("--library-only", action="store_true", help="libdlf.so alone, without the module on PyTorch's tensors")
    print(build(force=True, library_only=parser.parse_args().library_only))
