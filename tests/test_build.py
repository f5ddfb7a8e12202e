"""The build refuses a compiler that gives the grouped products fewer registers than their warps deal out among themselves."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def build():
    spec = importlib.util.spec_from_file_location("dip_build", os.path.join(ROOT, "paper_2412_01380_b200", "build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def log(registers):
    """What the assembler says of the kernels (8-bit, gate/up, kind): registers."""
    lines = ["ptxas info    : 0 bytes gmem"]
    for (fp8, gated, kind), n in registers.items():
        name = "_ZN43_GLOBAL__N__0_10_grouped_cu_015grouped_kernelINS_4KindILb%dELb%dELi%dEEEEEv14CUtensorMap_st" % (fp8, gated, kind)
        lines += ["ptxas info    : Compiling entry function '%s' for 'sm_100a'" % name, "ptxas info    : Function properties for %s" % name,
                  "    0 bytes stack frame, 0 bytes spill stores, 0 bytes spill loads", "ptxas info    : Used %d registers, used 5 barriers" % n]
    return "\n".join(lines)


ENOUGH = {(fp8, gated, kind): (120 if kind == 0 else 168 if fp8 else 96) for fp8 in (0, 1) for gated in (0, 1) for kind in (0, 1, 2)}


def test_enough_registers(build):
    build.check_registers(log(ENOUGH))
    build.check_registers(log({**ENOUGH, (0, 0, 0): 40}))         # (a kernel that deals none out)


@pytest.mark.parametrize("short", [(0, 1, 1), (0, 0, 2), (1, 0, 1), (1, 1, 2)])
def test_too_few_registers(build, short):
    with pytest.raises(RuntimeError):
        build.check_registers(log({**ENOUGH, short: ENOUGH[short] - 8}))


def test_a_log_without_the_kernels_proves_nothing(build):
    for kernels in ({}, {k: n for k, n in ENOUGH.items() if k != (1, 1, 2)}):
        with pytest.raises(RuntimeError):
            build.check_registers(log(kernels))


def test_the_numbers_are_those_of_the_source(build):
    """(few warps' share x 4 + the others' x how many) / all, of the kinds that deal registers out."""
    import re
    text = open(os.path.join(ROOT, "paper_2412_01380_b200", "csrc", "grouped.cu")).read()
    few = re.search(r"REGS_FEW = FP8 \? \(PAIR \? (\d+) : (\d+)\) : (\d+), REGS_MANY = FP8 \? \(PAIR \? (\d+) : (\d+)\) : (\d+)", text)
    pair8, whole8, bf16, pair8m, whole8m, bf16m = map(int, few.groups())
    assert re.search(r"OUT_WARPS = FP8 \|\| FEW \? 8 : 16", text)
    assert build.GROUPED_REGISTERS == {"1": max(pair8 * 4 + pair8m * 8, whole8 * 4 + whole8m * 8) // 12, "0": (bf16 * 4 + bf16m * 16) // 20}
