"""Builds libctc.so (the C ABI of include/ctc.h) for gfx950 with hipcc, and
_binding.so (the operators' Python binding, host code) with g++ and torch's
headers.  Networks need libctc.so alone (``--library``).

Every HIP source is compiled with packed-FP32 instruction selection turned
off; the host runtime and the kernels link into one shared library that
stays in this directory (no install step).
"""
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SO = os.path.join(HERE, "libctc.so")
SOURCES = [os.path.join(HERE, "csrc", "ctc_api.cpp"),
           os.path.join(HERE, "csrc", "ops_api.cpp"),
           os.path.join(HERE, "csrc", "library.hip")]
BINDING = os.path.join(HERE, "_binding.so")
BINDING_SOURCE = os.path.join(HERE, "csrc", "binding.cpp")
ARCH = "gfx950"


def hipcc():
    p = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc")
    return p if os.path.exists(p) else "hipcc"


def build(verbose=False, binding=True):
    """libctc.so and, unless not wanted, _binding.so; returns libctc.so."""
    tmp = "%s.tmp%d" % (SO, os.getpid())
    cmd = [hipcc(), "--offload-arch=" + ARCH, "-mcode-object-version=5",
           "-O3", "-std=c++17", "-fPIC",
           "-shared", "-Wall", "-Wno-unused-function",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-o", tmp] + SOURCES
    _run(cmd, verbose)
    os.replace(tmp, SO)
    if binding:
        build_binding(verbose)
    return SO


def build_binding(verbose=False):
    """Compiled against torch's headers and the libctc.so beside it."""
    import torch
    torch_dir = os.path.dirname(torch.__file__)
    tmp = "%s.tmp%d" % (BINDING, os.getpid())
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi(),
           BINDING_SOURCE, "-I", os.path.join(torch_dir, "include"), "-I",
           os.path.join(torch_dir, "include", "torch", "csrc", "api",
                        "include"),
           "-I", sysconfig.get_paths()["include"],
           "-L", os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch",
           "-ltorch_cpu", "-lc10", "-L", HERE, "-l:libctc.so",
           "-Wl,-rpath,$ORIGIN", "-o", tmp]
    _run(cmd, verbose)
    os.replace(tmp, BINDING)
    return BINDING


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    msgs = [ln for ln in (r.stdout + r.stderr).splitlines()
            if "packed-fp32-ops" not in ln]
    if r.returncode != 0:
        raise RuntimeError("%s failed:\n" % cmd[0] + "\n".join(msgs))
    if verbose and msgs:
        print("\n".join(msgs))


if __name__ == "__main__":
    build(verbose="-v" in sys.argv, binding="--library" not in sys.argv)
    print(SO)
