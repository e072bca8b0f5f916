"""The norm kernels that the library holds are those that some call reaches, and every call has its kernel (needs no GPU):
the rule of csrc/norm_plan.h, walked over widths and row counts, against the kernels' names in the built library."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2602_12529_amd import _lib, build

PROGRAM = r"""
#include <cstdio>
#include "norm_plan.h"
int main() {
  for (int forward = 0; forward < 2; ++forward)
    for (int64_t rows : {1, 2048, 2049, 1 << 27})
      for (int64_t H = 1; H <= 12400; ++H) {
        const ff::RowPlanH p = ff::row_plan_h(rows, H, forward != 0);
        if (p.ni > 0 && H > int64_t(8) * p.tpr * p.ni) return 1;   // columns that no thread takes
        std::printf("%d %d %d\n", forward, p.tpr, p.ni);
      }
}
"""


@pytest.fixture(scope="module")
def reached(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-I", build.CSRC, str(d / "plan.cpp"), "-o", str(d / "plan")], check=True)
    out = subprocess.run([str(d / "plan")], check=True, capture_output=True, text=True).stdout
    return {tuple(map(int, line.split())) for line in out.splitlines()}


@pytest.mark.parametrize("forward,kernel", [(1, "norm_affine_kernel"), (0, "norm_grad_kernel")])
def test_kernels_are_those_that_calls_reach(reached, forward, kernel):
    with open(_lib.LIB_PATH, "rb") as f:
        names = re.findall(rb"%sILb([01])ELi(\d+)ELi(\d+)ELb([01])E" % kernel.encode(), f.read())
    want = {(t, n) for way, t, n in reached if way == forward and n > 0}
    assert len(want) == 15 + forward
    for bf16 in (b"0", b"1"):
        for vec in (b"0", b"1"):
            built = {(int(t), int(n)) for b, t, n, v in names if (b, v) == (bf16, vec)}
            assert built == want, (kernel, bf16, vec, built ^ want)


def test_wide_rows_have_kernels_of_their_own(reached):
    assert {(t, n) for _, t, n in reached if n == 0} == {(512, 0)}
