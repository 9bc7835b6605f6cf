"""Build the HIP/C++ library ``libppconv.so`` in-tree for gfx950.

    python -m paper_2004_11250_amd.build            # build (always recompiles)
    python -m paper_2004_11250_amd.build --host     # also the g++-only packer library

Every HIP translation unit is compiled with packed-FP32 instructions disabled
(``-Xclang -target-feature -Xclang -packed-fp32-ops``); the host pass warns
that it does not know the feature, which is harmless.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libppconv.so")
HOST_LIB = os.path.join(PKG, "libppconv_host.so")
CEIL_LIB = os.path.join(PKG, "libppceil.so")
TENSORS_LIB = os.path.join(PKG, "_tensors.so")
OBJDIR = os.path.join(PKG, "_build")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
# -structurizecfg-skip-uniform-regions: the pattern dispatch of the pruned
# conv is a wave-uniform branch tree; left unstructurized it needs no
# accumulator copies at the joins (the structurized form duplicates them).
# -simplifycfg-sink-common=false: otherwise the eight pattern cases, which
# have the same shape, are merged into one FMA block fed by register copies.
HIP_FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-Xclang", "-target-feature",
             "-Xclang", "-packed-fp32-ops", "-mllvm", "-structurizecfg-skip-uniform-regions",
             "-mllvm", "-simplifycfg-sink-common=false", "-Wno-pass-failed", f"-I{INCLUDE}", f"-I{CSRC}"]


def _run(cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"command failed ({r.returncode}): {' '.join(cmd)}\n{out}")
    return out


# the kernel headers the run-time compiler (jit.cpp) builds specialised
# kernels from, embedded as string literals
JIT_HEADERS = (("conv_pp_wave.hpp", CSRC), ("conv_pp_kernel.hpp", CSRC), ("conv_pp.hpp", CSRC), ("pp.h", INCLUDE))


def write_jit_sources() -> None:
    lines = ["// generated by build.py: the kernel headers, for run-time compilation", ""]
    texts = []
    for name, d in JIT_HEADERS:
        with open(os.path.join(d, name)) as fh:
            text = fh.read()
        if ")PPJIT" in text:
            raise RuntimeError(f"{name} contains the raw-string delimiter")
        texts.append(text)
    lines.append(f"static const int kJitHeaderCount = {len(JIT_HEADERS)};")
    lines.append("static const char* const kJitHeaderNames[] = {" +
                 ", ".join(f'"{n}"' for n, _ in JIT_HEADERS) + "};")
    lines.append("static const char* const kJitHeaders[] = {")
    for t in texts:
        lines.append('R"PPJIT(' + t + ')PPJIT",')
    lines.append("};")
    tmp = os.path.join(OBJDIR, "jit_sources.inc.tmp")
    with open(tmp, "w") as fh:
        fh.write("\n".join(lines) + "\n")
    os.replace(tmp, os.path.join(OBJDIR, "jit_sources.inc"))


def build(verbose: bool = False) -> str:
    os.makedirs(OBJDIR, exist_ok=True)
    write_jit_sources()
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.cpp")))
    objs = []
    jobs = []
    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        for s in srcs:
            o = os.path.join(OBJDIR, os.path.basename(s) + ".o")
            objs.append(o)
            cmd = [HIPCC] + HIP_FLAGS + [f"-I{OBJDIR}"] + (["-x", "hip"] if s.endswith(".hip") else []) + \
                ["-c", s, "-o", o]
            jobs.append(ex.submit(_run, cmd))
        for j in jobs:
            out = j.result()
            if verbose and out.strip():
                print(out)
    tmp = LIB + ".tmp"
    _run([HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp] + objs + ["-lhiprtc", "-ldl"])
    os.replace(tmp, LIB)
    build_ceiling()
    build_tensors()
    return LIB


def build_tensors():
    """The binding's Python module of calls with native checks (torch's and Python's
    headers; the library itself knows nothing of either).  Where those are missing it
    is left out with a note, and None: the library is whole without it, and the calls
    that need the module say that it is not built."""
    import sysconfig

    headers = sysconfig.get_paths()["include"]
    try:
        import torch
        missing = None if os.path.exists(os.path.join(headers, "Python.h")) else f"{headers}/Python.h"
    except ImportError:
        missing = "torch"
    if missing:
        if os.path.exists(TENSORS_LIB):
            os.remove(TENSORS_LIB)      # (of other sources, perhaps)
        print(f"{os.path.basename(TENSORS_LIB)} is not built: no {missing}", file=sys.stderr)
        return None
    at = os.path.dirname(torch.__file__)
    tmp = TENSORS_LIB + ".tmp"
    _run([HIPCC, "-x", "c++", "-no-hip-rt", "-O2", "-std=c++17", "-fPIC", "-shared", f"-I{at}/include", f"-I{at}/include/torch/csrc/api/include",
          f"-I{headers}", f"-I{INCLUDE}", os.path.join(PKG, "binding", "tensors.cpp"), "-o", tmp,
          f"-L{at}/lib", "-ltorch_python", "-ltorch_cpu", "-lc10"])
    os.replace(tmp, TENSORS_LIB)
    return TENSORS_LIB


def build_ceiling() -> str:
    """The measured-ceiling micro-benchmarks the benchmark reports beside the
    published peaks (a library of its own: it allocates and synchronises)."""
    tmp = CEIL_LIB + ".tmp"
    _run([HIPCC] + HIP_FLAGS + ["-shared", "-x", "hip", os.path.join(PKG, "ceiling", "ceiling.hip"), "-o", tmp])
    os.replace(tmp, CEIL_LIB)
    return CEIL_LIB


def build_host() -> str:
    """The packer, the pruning projections and blob validation alone, built
    with g++ (no HIP)."""
    tmp = HOST_LIB + ".tmp"
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-I{INCLUDE}", f"-I{CSRC}",
          os.path.join(CSRC, "pack.cpp"), os.path.join(CSRC, "project.cpp"), "-o", tmp])
    os.replace(tmp, HOST_LIB)
    return HOST_LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
    if "--host" in sys.argv:
        print(build_host())
