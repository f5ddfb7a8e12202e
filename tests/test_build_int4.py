"""The build refuses a compiler that gives the 4-bit products of many rows fewer registers than their warps deal out among themselves."""
import os
import re

import pytest

from test_build import ROOT, build  # noqa: F401


def log(registers):
    """What the assembler says of the kernels (gate/up): registers."""
    lines = ["ptxas info    : 0 bytes gmem"]
    for gated, n in registers.items():
        name = "_ZN45_GLOBAL__N__0_12_int4_many_cu_016int4_many_kernelINS_8ManyKindILb%dEEEEEv14CUtensorMap_stS3_S3_NS_13GroupedParamsE" % gated
        lines += ["ptxas info    : Compiling entry function '%s' for 'sm_100a'" % name, "ptxas info    : Function properties for %s" % name,
                  "    0 bytes stack frame, 20 bytes spill stores, 56 bytes spill loads", "ptxas info    : Used %d registers, used 4 barriers" % n]
    return "\n".join(lines)


def test_enough_registers(build):  # noqa: F811
    build.check_int4_many_registers(log({0: 128, 1: 126}))


@pytest.mark.parametrize("kernels", [{0: 120, 1: 128}, {0: 128, 1: 125}, {0: 128}, {}])
def test_too_few_registers_or_a_log_without_the_kernels(build, kernels):  # noqa: F811
    with pytest.raises(RuntimeError):
        build.check_int4_many_registers(log(kernels))


def test_the_source_is_checked_by_the_number_it_needs(build):  # noqa: F811
    """(a share for four warps, another for four, the third for the others) / all: every file that deals registers out has a check."""
    folder = os.path.join(ROOT, "paper_2412_01380_b200", "csrc")
    text = open(os.path.join(folder, "int4_many.cu")).read()
    few, codes, many = map(int, re.search(r"REGS_FEW = (\d+), REGS_CODES = (\d+), REGS_MANY = (\d+)", text).groups())
    out = int(re.search(r"OUT_WARPS = (\d+)", text).group(1))
    assert build.INT4_MANY_REGISTERS == -(-(few * 4 + codes * 4 + many * out) // (8 + out))
    deal = {f for f in os.listdir(folder) if "setmaxnreg" in open(os.path.join(folder, f)).read()}
    assert deal == set(build.REGISTER_CHECKS)
