"""CPU-only: which way the logits of a token's entries come, and how many threads go through a row, of the calls that the GPU tests make
(csrc/loss_plan.hpp, compiled here without a GPU): every pair of the two has to be reached.  And the sizes of pieces."""
import os
import shutil
import subprocess

import pytest

from test_gpu_loss import FEW, LARGER, PICKED, SIZES
from test_gpu_loss_entries import FROM_TILES, SCORES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <stdio.h>
#include "loss_plan.hpp"
using namespace tsenor_dev;
int main() {
  LossShape s = {};
  long tokens, vocab, width;
  int bf16, gradients, teacher;
  while (scanf("%ld %ld %ld %d %d %d %d", &tokens, &vocab, &width, &bf16, &gradients, &s.k, &teacher) == 7) {
    s.tokens = tokens, s.vocab = vocab, s.width = width, s.bf16 = bf16, s.dh = s.dweight = gradients, s.teacher = teacher;
    s.in_place = bf16 && width % 8 == 0, s.states_too = width % 64 == 0;
    const LossPlan p = loss_plan(s);
    printf("%ld:%s:%s:%d\n", (long)p.rows, p.few ? "few" : p.direct ? "direct" : "gathered", s.k == 1 ? "one" : p.picked ? "ordered" : "looked", p.row_threads);
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """(rows of a piece, words about the plan) of calls (tokens, vocab, width, bf16, gradients, k, teacher)"""
    folder = tmp_path_factory.mktemp("plan")
    (folder / "plan.cpp").write_text(PROGRAM)
    compiler = shutil.which("g++") or shutil.which("c++")
    subprocess.run([compiler, "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2505_23949_amd", "csrc"), "-o", folder / "plan",
                    folder / "plan.cpp"], check=True)

    def plans_of(calls):
        text = "".join(" ".join(str(int(v)) for v in c) + "\n" for c in calls)
        lines = subprocess.run([folder / "plan"], input=text, capture_output=True, text=True, check=True).stdout.split()
        return [(int(line.split(":", 1)[0]), line.split(":", 1)[1]) for line in lines]

    return plans_of


def test_every_way_of_the_entries_is_tested(plans):
    calls = [(*s, dtype == "bf16", 1, k, teacher) for s in SIZES + FEW for dtype in ("bf16", "f32") for k, teacher in ((1, 0), (1, 1), (min(s[1], 5), 1), (min(s[1], 70), 1))]
    calls += [(t, v, w, b, 1, 1, 0) for t, v, w, dh, dweight in LARGER if dh or dweight for b in (0, 1)]
    calls += [(t, v, w, dtype == "bf16", 1, k, 1) for t, v, w, dtype, k, _ in PICKED] + [(t, v, w, dtype == "bf16", 1, k, 1) for t, v, w, dtype, k in FROM_TILES]
    calls += [(t, v, w, dtype == "bf16", 0, k, 1) for t, v, w, dtype, k in SCORES]
    got = {words for _, words in plans(calls)}
    want = {f"gathered:{way}:{threads}" for way in ("one", "ordered") for threads in (64, 256, 1024)}
    want |= {"few:one:256", "few:looked:256", "few:one:1024", "few:looked:1024", "direct:one:256", "direct:looked:256", "direct:looked:1024"}
    assert want <= got, sorted(want - got)


def test_pieces_fit_a_launch(plans):
    """A grid has fewer than 2^32 threads, and each row of a piece takes 256 of them (1024 only where rows are few)."""
    calls = [(tokens, vocab, width, bf16, gradients, k, 1) for tokens in (1 << 24, (1 << 24) - 1, 5000000) for vocab in (1, 64, 65, 300) for width in (1, 64)
             for bf16 in (0, 1) for gradients in (0, 1) for k in (1, 4)]
    for call, (rows, words) in zip(calls, plans(calls)):
        assert (rows + 63) // 64 * 64 * max(256, int(words.split(":")[-1])) < 1 << 32, call
