"""CPU-only: how the calls that the GPU tests make are made (csrc/loss_plan.hpp, compiled here without a GPU).  They have to reach every
kernel, so a change of the costs that moves a shape to another one is to be seen here."""
import os
import shutil
import subprocess

import pytest

from test_gpu_loss import FEW, LARGER, PICKED, SIZES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <stdio.h>
#include "loss_plan.hpp"
using namespace tsenor_dev;
const char* const names[] = {"none", "few", "small", "tile", "pairs", "wide", "large"};
void tell(const char* what, const ProductPlan& p) { printf(" %s:%s%s", what, names[p.kind], p.splits > 1 ? "+" : ""); }
int main() {
  LossShape s = {};
  long tokens, vocab, width;
  int bf16, dh, dweight, teacher, in_place, states_too;
  while (scanf("%ld %ld %ld %d %d %d %d %d %d %d", &tokens, &vocab, &width, &bf16, &dh, &dweight, &s.k, &teacher, &in_place, &states_too) == 10) {
    s.tokens = tokens, s.vocab = vocab, s.width = width;
    s.bf16 = bf16, s.dh = dh, s.dweight = dweight, s.teacher = teacher, s.in_place = in_place, s.states_too = states_too;
    const LossPlan p = loss_plan(s);
    if (p.few) printf(" few"); else tell("logits", p.logits);
    if (p.both.use) {
      tell("both_dh", p.both.dh), tell("both_dweight", p.both.dweight);
    } else {
      if (p.few_dh) printf(" few_dh%s%s", p.dh_of_few.splits > 1 ? "+" : "", p.dh_of_few.words > kFewDhWords ? "long" : "");
      else if (dh) tell("dh", p.dh);
      for (int k = 0; k < p.dweight.count; ++k) tell(k ? "rest" : "dweight", p.dweight.parts[k]);
    }
    printf("%s%s%s%s rows:%ld\n", p.direct ? " direct" : "", p.counted ? " counted" : "", p.picked ? " picked" : "", tokens > p.rows ? " pieces" : "", (long)p.rows);
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
        text = "".join(" ".join(str(int(v)) for v in s) + "\n" for s in shapes)
        out = subprocess.run([folder / "plan"], input=text, capture_output=True, text=True, check=True).stdout
        return [line.split() for line in out.splitlines()]

    return plans_of


def shape(tokens, vocab, width, dtype="bf16", dh=True, dweight=True, k=1, teacher=False):
    bf16 = dtype == "bf16"
    return (tokens, vocab, width, bf16, dh, dweight, k, teacher, bf16 and width % 8 == 0, width % 64 == 0)


def test_every_kernel_is_reached_by_a_tested_call(plans):
    calls = [shape(*s, dtype) for s in SIZES for dtype in ("bf16", "f32")]
    calls += [shape(*s, dtype) for s in FEW for dtype in ("bf16", "f32")]
    calls += [shape(t, v, w, dh=dh, dweight=dweight) for t, v, w, dh, dweight in LARGER]
    calls += [shape(t, v, w, dtype, k=k, teacher=True) for t, v, w, dtype, k, _ in PICKED]
    calls += [shape(t, 700, 192, dh=False, dweight=False) for t in (1, 7, 40, 300)]            # outputs that are wanted
    calls += [shape(538, 40884, 72, dweight=False), shape(9000, 131072, 64), shape(9000, 131072, 64, "f32")]  # dh alone, pieces
    got = {word for line in plans(calls) for word in line}
    kinds = ("small", "tile", "pairs", "wide", "large")
    want = {f"logits:{k}" for k in kinds} | {"logits:small+"}
    want |= {f"{p}:{k}{split}" for p in ("dh", "dweight") for k in kinds for split in ("", "+")} | {"rest:small", "rest:small+", "rest:tile+", "rest:pairs"}
    want |= {f"both_{p}:{k}" for p in ("dh", "dweight") for k in ("small", "tile")} | {"both_dh:small+", "both_dh:tile+", "both_dweight:small+"}
    want |= {"few_dh", "few_dh+", "few_dh+long"}
    want |= {"few", "direct", "counted", "picked", "pieces"}
    assert want <= got, sorted(want - got)


def test_pieces_are_bounded(plans):
    for vocab, dtype, size in ((131072, "bf16", 2), (131072, "f32", 10), (1 << 21, "bf16", 2), (100, "bf16", 2)):
        for tokens in (1, 1000, 100000, 1 << 24):
            line = plans([shape(tokens, vocab, 64, dtype)])[0]
            rows = int(line[-1].split(":")[1])
            assert rows * vocab * size <= max(2 ** 31, 256 * vocab * size) + 64 * rows * size
            assert rows >= min(tokens, 256) and (rows % 256 == 0 or rows >= tokens)


def test_a_call_without_work_has_a_plan(plans):
    for s in (shape(0, 100, 64), shape(5, 0, 64), shape(5, 100, 0), shape(0, 0, 0)):
        assert plans([s])[0]
