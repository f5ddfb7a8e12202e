"""Build the CUDA library in-tree: paper_2412_01380_b200/libdip.so (sm_100a only).

Each .cu file is compiled to an object of its own (in parallel, and only when it or a header
is newer than the object), then the objects are linked into the shared library.
"""
import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libdip.so")
SOURCES = ["api.cu", "topk.cu", "gemv.cu", "gemv_fused.cu", "gemv_direct_bt.cu", "gemv_int4.cu", "gemv_tc.cu", "gemv_noalloc.cu", "pack.cu", "tier.cu", "rowdot.cu",
           "experts.cu", "route.cu", "grouped.cu", "int4_few.cu", "int4_many.cu", "sample.cu"]
HEADERS = [os.path.join(CSRC, "common.cuh"), os.path.join(CSRC, "gemv_common.cuh"), os.path.join(CSRC, "select_core.cuh"), os.path.join(CSRC, "cache_update.cuh"), os.path.join(CSRC, "float8.cuh"), os.path.join(CSRC, "int4_codes.cuh"), os.path.join(CSRC, "grouped_common.cuh"), os.path.join(ROOT, "include", "dip.h")]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]

# Registers per thread that a launch of the grouped products must have (8-bit: "1"), because their warps deal them out again: with fewer the
# warps that take more would wait for ever, and every launch is refused.
GROUPED_REGISTERS = {"1": 168, "0": 96}
INT4_MANY_REGISTERS = 126                       # the same of the 4-bit products of many rows


def check_registers(log: str) -> None:
    """log: what ptxas -v says of grouped.cu.  Kind<8 bits, gate/up, kind>; kind 0 (few rows) deals none out."""
    found = re.findall(r"Compiling entry function '[^']*grouped_kernel[^']*KindILb([01])ELb([01])ELi([0-2])E.*?Used (\d+) registers", log, re.S)
    short = ["%s of %d" % (f, GROUPED_REGISTERS[f[0]]) for f in found if f[2] != "0" and int(f[3]) < GROUPED_REGISTERS[f[0]]]
    if len(found) != 12 or short:
        raise RuntimeError("grouped.cu: %d of 12 kernels, too few registers in (8 bits, gate/up, kind, registers): %s" % (len(found), short))


def check_int4_many_registers(log: str) -> None:
    """log: what ptxas -v says of int4_many.cu.  ManyKind<gate/up>."""
    found = re.findall(r"Compiling entry function '[^']*int4_many_kernel[^']*ManyKindILb([01])E.*?Used (\d+) registers", log, re.S)
    short = [f for f in found if int(f[1]) < INT4_MANY_REGISTERS]
    if len(found) != 2 or short:
        raise RuntimeError("int4_many.cu: %d of 2 kernels, fewer than %d registers in (gate/up, registers): %s" % (len(found), INT4_MANY_REGISTERS, short))


REGISTER_CHECKS = {"grouped.cu": check_registers, "int4_many.cu": check_int4_many_registers}


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def up_to_date() -> bool:
    return not _stale(LIB, [os.path.join(CSRC, s) for s in SOURCES] + HEADERS)


def _compile(src: str, force: bool, verbose: bool) -> str:
    path = os.path.join(CSRC, src)
    obj = os.path.join(OBJ, src[:-3] + ".o")
    if force or _stale(obj, [path] + HEADERS):
        tmp = obj + ".tmp.%d" % os.getpid()
        check = REGISTER_CHECKS.get(src)
        cmd = [_nvcc(), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose or check else []), "-c", path, "-o", tmp]
        done = subprocess.run(cmd, stderr=subprocess.PIPE if check else None, text=True)
        if check and (verbose or done.returncode):
            sys.stderr.write(done.stderr)
        done.check_returncode()
        if check:
            check(done.stderr)
        os.replace(tmp, obj)
    return obj


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and up_to_date():
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        objs = list(pool.map(lambda s: _compile(s, force, verbose), SOURCES))
    tmp = LIB + ".tmp.%d" % os.getpid()
    subprocess.run([_nvcc(), "-shared", "-cudart", "static", "-gencode", "arch=compute_100a,code=sm_100a",
                    *objs, "-o", tmp], check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
