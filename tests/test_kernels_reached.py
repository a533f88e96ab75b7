"""The library holds no kernel that no call launches, and none that would refuse to start: names and registers of its own kernels."""
import re
import subprocess

import pytest

from paper_2605_01989_b200 import binding as dblp
from paper_2605_01989_b200 import build as lib_build

OPERAND = re.compile(r"k_rows_(?:wide|long)<(__half|__nv_bfloat16), \d, dblp::Epi\w+<(__half|__nv_bfloat16)")


def kernels(name):
    text = subprocess.run(["nm", "-C", dblp.LIB_PATH], check=True, capture_output=True, text=True).stdout
    return {line.split(" ", 2)[2] for line in text.splitlines() if "void dblp::%s<" % name in line}


def test_kernels_for_few_rows_have_one_operand_type():
    found = kernels("k_rows_wide") | kernels("k_rows_long")
    types = [OPERAND.search(k).groups() for k in found]
    assert types and all(a == b for a, b in types)


def test_only_sums_that_may_be_empty_have_a_kernel_for_it():
    found = kernels("k_product_none")
    assert found and not [k for k in found if "EpiLast" in k or "EpiPoly" in k]


def test_the_build_looks_at_the_registers_that_runs_count_on():
    found = lib_build.registers()
    runs = [name for name in found if "k_productILi2ELb1E" in name]
    assert len(runs) >= 6 and len(found) > 100
    lib_build.check_registers(found)
    with pytest.raises(RuntimeError, match="160"):
        lib_build.check_registers({**found, runs[0]: 160})
    lib_build.check_registers({**found, runs[0].replace("Lb1E", "Lb0E"): 160})
