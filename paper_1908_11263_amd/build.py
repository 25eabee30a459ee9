"""Build the gfx950 library ``libqnn.so`` in-tree with hipcc.

Every HIP source under csrc/ is compiled for gfx950 only and linked into one
shared library next to this file.  Packed-FP32 instruction generation is
switched off for all device code.  The compiled part of the binding
(csrc/lm_bind.cpp) is host code for torch's C++ headers: a module of its own,
``_lm_bind.so``.
"""
import concurrent.futures
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libqnn.so")
BINDING = os.path.join(HERE, "_lm_bind.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I" + INCLUDE, "-I" + CSRC,
]


# per-source extra flags: the whole-image kernels keep their MFMA
# accumulators in ordinary VGPRs (their epilogues read them right away, and
# the accumulation registers would cost copies and occupancy), and their
# twelve leading scalar arguments are preloaded into scalar registers
_IMG = ["-mllvm", "-amdgpu-mfma-vgpr-form", "-mllvm", "-amdgpu-kernarg-preload-count=12"]
# the classifier kernel's eight scalar arguments likewise
EXTRA = {"conv_img_p4.hip": _IMG, "conv_img_p16.hip": _IMG, "conv_img_p32.hip": _IMG,
         "linear.hip": ["-mllvm", "-amdgpu-kernarg-preload-count=8"]}


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".hip"))


def _compile(src):
    obj = os.path.join(BUILD, os.path.basename(src)[:-4] + ".o")
    cmd = [HIPCC] + FLAGS + EXTRA.get(os.path.basename(src), []) + ["-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s%s" % (src, r.stdout, r.stderr))
    return obj


def build_binding():
    """Compile the host's path of lm.py's calls (csrc/lm_bind.cpp) against torch's headers."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    rocm = os.path.dirname(os.path.dirname(HIPCC))
    tmp = BINDING + ".tmp%d" % os.getpid()
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-Wno-sign-compare",
           "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), "-I" + INCLUDE,
           "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(rocm, "include")]
    for path in cpp_extension.include_paths():
        cmd += ["-isystem", path]
    cmd += [os.path.join(CSRC, "lm_bind.cpp"), "-o", tmp]
    for path in cpp_extension.library_paths():
        cmd += ["-L" + path, "-Wl,-rpath," + path]
    cmd += ["-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for lm_bind.cpp:\n%s%s" % (r.stdout, r.stderr))
    os.replace(tmp, BINDING)
    return BINDING


def build(jobs=None, verbose=True):
    """Compile every HIP source, link libqnn.so and build the binding (always recompiles)."""
    os.makedirs(BUILD, exist_ok=True)
    srcs = sources()
    jobs = jobs or min(len(srcs), max(1, (os.cpu_count() or 2) // 2))
    with concurrent.futures.ThreadPoolExecutor(jobs) as ex:
        binding = ex.submit(build_binding)
        objs = list(ex.map(_compile, srcs))
        binding.result()
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s%s" % (r.stdout, r.stderr))
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB, file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build()
