"""Build libjq.so (the gfx950 HIP library behind include/jq.h and jq_block.h) in-tree with hipcc.

Each source compiles to its own object in parallel (_build/), then one hipcc
link makes the shared library.  Every call compiles every source.  Alongside,
the BF6 kernels are compiled to device assembly once more and the GEMM's
hand-ordered vector loads are checked against their waits (check_waits.py); a
failed check fails the build.
"""

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

try:
    from . import check_waits
except ImportError:  # run as a script
    import check_waits

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ_DIR = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libjq.so")
SOURCES = ["quantize.hip", "ternary.hip", "gemm.hip", "gemm_narrow.hip", "gemm_wide.hip", "gemm_group.hip", "f6.hip",
           "f6_narrow.hip", "f6_narrow_group.hip", "f6_quant_few.hip", "jq_api.cpp", "rmsnorm.hip", "fp8_quant.hip",
           "fp8_gemm.hip", "rope_append.hip", "paged_attention.hip", "gated_act.hip", "prompt_attention.hip",
           "jq_block_api.cpp"]
# The compiled half of the binding of jq_block.h: a Python extension on torch's C++ headers.
BINDING_SOURCE = "jq_block_py.cpp"
BINDING = os.path.join(PKG, "_jq_block.so")
ARCH = "gfx950"

# Per-source flags: the BF6 and 8-bit GEMMs are built without machine sinking, which
# would move the first k-step's MFMAs of a BF6 stage below its barrier, and the
# multiply-adds of an 8-bit stage behind all of its MFMAs (100 registers spilled).
SOURCE_FLAGS = {"f6.hip": ["-mllvm", "-disable-machine-sink"], "fp8_gemm.hip": ["-mllvm", "-disable-machine-sink"]}
# Sources whose asm-issued loads are checked against their waits, and the
# kernel names checked in each.
CHECKED_SOURCES = {"f6.hip": "w4a4_f6_gemm_kernel", "fp8_gemm.hip": "fp8_gemm_kernel",
                   "paged_attention.hip": "paged_attention_wide_kernel", "prompt_attention.hip": "prompt_attention_kernel"}

HIPCC_FLAGS = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-std=c++17",
    "-fPIC",
    # every fp32 operation of the quantiser and the epilogue is rounded on its own
    "-ffp-contract=off",
    # no packed-fp32 VALU instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall",
]


def hipcc():
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: the HIP library cannot be built")


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}): {' '.join(cmd)}\n{out}")
    if verbose and out.strip():
        print(out, flush=True)


def build(verbose=False, extra_flags=(), jobs=None):
    """Compile the library; returns the path of the built .so."""
    os.makedirs(OBJ_DIR, exist_ok=True)
    cc = hipcc()
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    objs = [os.path.join(OBJ_DIR, os.path.splitext(s)[0] + ".o") for s in SOURCES]
    cmds = [[cc, *HIPCC_FLAGS, *SOURCE_FLAGS.get(s, []), *extra_flags, *inc, "-c", os.path.join(CSRC, s), "-o", o]
            for s, o in zip(SOURCES, objs)]
    checked = [s for s in SOURCES if s in CHECKED_SOURCES]
    jobs = jobs or max(1, min(len(cmds) + len(checked), os.cpu_count() or 1))
    with ThreadPoolExecutor(max_workers=jobs) as pool:
        futs = [pool.submit(_run, c, verbose) for c in cmds]
        futs += [pool.submit(check_waits.compile_and_check,
                             [cc, *HIPCC_FLAGS, *SOURCE_FLAGS.get(s, []), *extra_flags, *inc],
                             os.path.join(CSRC, s), os.path.join(OBJ_DIR, os.path.splitext(s)[0] + ".s"),
                             CHECKED_SOURCES[s])
                 for s in checked]
        for f in futs:
            f.result()
    tmp = LIB + ".tmp"
    _run([cc, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp], verbose)
    os.replace(tmp, LIB)
    build_binding(verbose)
    return LIB


def binding_lacks():
    """What jq_block.py's extension needs and this machine does not have, or None."""
    import sysconfig

    try:
        import torch
    except ImportError:
        return "torch is not installed"
    if torch.version.hip is None:
        return "torch is not built for ROCm"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python.h is not installed"
    return None


def build_binding(verbose=False):
    """Compile jq_block.py's extension against the built libjq.so; returns its path.

    libjq.so and its C ABI need none of what the extension needs: where that is missing, says so and returns None, and
    jq_block.py raises at its first call."""
    import sysconfig

    lacks = binding_lacks()
    if lacks is not None:
        if os.path.exists(BINDING):  # of an earlier build
            os.remove(BINDING)
        print(f"{os.path.basename(BINDING)} not built: {lacks}", flush=True)
        return None
    from torch.utils import cpp_extension

    rocm = os.path.dirname(os.path.dirname(hipcc()))
    dirs = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], os.path.join(rocm, "include"),
                                            os.path.join(ROOT, "include")]
    cxx = shutil.which("g++")
    tmp = BINDING + ".tmp"
    _run([*([cxx] if cxx else [hipcc(), "-x", "c++"]), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
          "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM", *[a for d in dirs for a in ("-isystem", d)],
          os.path.join(CSRC, BINDING_SOURCE), "-o", tmp,
          "-L", PKG, "-ljq", *[a for d in cpp_extension.library_paths() for a in ("-L", d)],
          "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_hip", "-ltorch_python", "-Wl,-rpath,$ORIGIN"], verbose)
    os.replace(tmp, BINDING)
    return BINDING


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
