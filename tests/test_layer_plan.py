"""CPU-only: which kernels a product is given to (csrc/layer_plan.hpp, compiled here without a GPU).  The shapes that the GPU tests multiply
have to reach every one of them, so a change of the costs that moves a shape to another kernel is to be seen here."""
import os
import shutil
import subprocess

import pytest

from test_gpu_layer_products import PRODUCTS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <stdio.h>
#include "layer_plan.hpp"
int main() {
  const char* const names[] = {"none", "few", "small", "tile", "pairs", "wide", "large"};
  long m, n, k;
  while (scanf("%ld %ld %ld", &m, &n, &k) == 3) {
    const tsenor_dev::Plan p = tsenor_dev::plan_of(m, n, (k + 127) / 128);
    printf("%zu", p.workspace);
    for (int i = 0; i < p.count; ++i) {
      const tsenor_dev::Part& a = p.parts[i];
      printf(" %s%s %ld %ld %ld %ld", names[a.kind], a.splits > 1 ? "+" : "", (long)a.m0, (long)a.n0, (long)a.m, (long)a.n);
    }
    printf("\n");
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    folder = tmp_path_factory.mktemp("plan")
    (folder / "plan.cpp").write_text(PROGRAM)
    compiler = shutil.which("g++") or shutil.which("c++")
    subprocess.run([compiler, "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2505_23949_amd", "csrc"), "-o", folder / "plan",
                    folder / "plan.cpp"], check=True)

    def plans_of(shapes):
        text = "".join("%d %d %d\n" % s for s in shapes)
        lines = subprocess.run([folder / "plan"], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        out = []
        for line in lines:
            words = line.split()
            parts = [(words[i], *map(int, words[i + 1:i + 5])) for i in range(1, len(words), 5)]
            out.append((int(words[0]), parts))
        return out

    return plans_of


def test_the_tested_products_reach_every_kernel(plans):
    for (m, n, k, kinds), (_, parts) in zip(PRODUCTS, plans([p[:3] for p in PRODUCTS])):
        assert tuple(p[0] for p in parts) == kinds, (m, n, k)
    reached = {kind for p in PRODUCTS for kind in p[3]}
    assert reached == {"few", "small", "small+", "tile", "pairs", "wide", "large"}


def test_the_parts_cover_the_product(plans):
    shapes = [(m, n, k) for m in (1, 16, 17, 100, 1999, 5000, 14331) for n in (1, 130, 4093, 9001, 28672) for k in (1, 300, 4100, 14336)]
    for (m, n, k), (workspace, parts) in zip(shapes, plans(shapes)):
        assert sum(p[3] * p[4] for p in parts) == m * n and 1 <= len(parts) <= 2
        assert parts[0][1:3] == (0, 0)
        if len(parts) == 2:  # what the first launch leaves, by rows of a or by rows of b; it begins at whole groups of scales
            (_, _, _, m1, n1), (_, m0, n0, m2, n2) = parts
            assert (m0, n0, m2, n2) in ((m1, 0, m - m1, n), (0, n1, m, n - n1)) and m0 % 16 == 0 and n0 % 16 == 0
        assert (workspace > 0) == any(p[0] == "small+" for p in parts)
