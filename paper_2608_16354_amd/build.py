"""Build the HIP library libdrivecache.so (gfx950) and the tensor binding _binding.so in-tree.

    python -m paper_2608_16354_amd.build

Device sources (*.hip) go through hipcc for gfx950; host sources (*.cpp) through
amdclang++ with -ffp-contract=off, so the schedule's floating-point arithmetic
is one IEEE operation at a time.  The binding (binding.cpp) is built against torch's headers; the
library needs neither it nor torch, and is installed before a binding that fails is reported.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libdrivecache.so")
BINDING = os.path.join(PKG, "_binding.so")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
ARCH = "gfx950"

HIPCC_FLAGS = ["-O3", "-fPIC", "-std=c++17", f"--offload-arch={ARCH}",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-ffp-contract=fast", "-Wall", "-Wno-unused-result"]
# per-file extra flags: keep MFMA results in VGPRs where the softmax or the blocks' scales read them
EXTRA_FLAGS = {f: ["-mllvm", "-amdgpu-mfma-vgpr-form=true"] for f in ("attention.hip", "gemm_f8.hip")}
HOST_FLAGS = ["-O2", "-fPIC", "-std=c++17", "-ffp-contract=off", "-D__HIP_PLATFORM_AMD__",
              f"-I{ROCM}/include", "-Wall"]


def _run(cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError("build step failed:\n" + " ".join(cmd) + "\n" + r.stdout)
    return r.stdout


def sources():
    return sorted(f for f in os.listdir(CSRC) if f.endswith((".hip", ".cpp")))


def _build_binding(clang):
    """What the compiler printed, or None where there is no torch to build against."""
    try:
        import torch
    except (ImportError, OSError) as e:
        print(f"the tensor binding is not built: no torch ({e})", file=sys.stderr)
        return None
    t = os.path.dirname(torch.__file__)
    return _run([clang, "-O2", "-fPIC", "-shared", "-std=c++17", "-Wall", "-D__HIP_PLATFORM_AMD__",
                 f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                 "-isystem", f"{t}/include", "-isystem", f"{t}/include/torch/csrc/api/include",
                 "-isystem", sysconfig.get_paths()["include"], f"-I{ROCM}/include",
                 os.path.join(PKG, "binding.cpp"), "-o", BINDING + ".tmp", f"-L{t}/lib", "-ltorch_python", "-ltorch_cpu",
                 "-lc10"])


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    hipcc = os.path.join(ROCM, "bin", "hipcc")
    clang = os.path.join(ROCM, "llvm", "bin", "clang++")
    jobs = []
    objs = []
    for f in sources():
        src = os.path.join(CSRC, f)
        obj = os.path.join(BUILD, f + ".o")
        objs.append(obj)
        if f.endswith(".hip"):
            jobs.append([hipcc, *HIPCC_FLAGS, *EXTRA_FLAGS.get(f, []), "-c", src, "-o", obj])
        else:
            jobs.append([clang, *HOST_FLAGS, "-c", src, "-o", obj])
    with ThreadPoolExecutor(max(1, min(8, os.cpu_count() or 1))) as ex:
        binding = ex.submit(_build_binding, clang)
        outs = list(ex.map(_run, jobs))
    if verbose:
        for o in outs:
            if o.strip():
                print(o)
    tmp = LIB + ".tmp"
    _run([hipcc, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp, *objs,
          f"-L{ROCM}/lib", "-lamdhip64"])
    os.replace(tmp, LIB)
    failure = binding.exception()
    if failure is None and binding.result() is not None:
        os.replace(BINDING + ".tmp", BINDING)
        if verbose and binding.result().strip():
            print(binding.result())
    elif os.path.exists(BINDING):               # it belongs to another library
        os.remove(BINDING)
    if failure is not None:
        raise RuntimeError(f"the library is built, the tensor binding is not: {failure}") from failure
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
