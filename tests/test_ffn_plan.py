"""The tiles and splits that the gated block's rule picks at the sizes of the GPU tests: a
change of the rule may not leave a kernel instance without one.  The rule is host
arithmetic in a header of its own, compiled here."""
import os
import shutil
import subprocess

import pytest

from _ffn_cases import CASES

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_03011_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "isoloco_ffn_plan.h"
using namespace isoloco;
int main() {
  long long m, d, f;
  int f32;
  while (std::scanf("%d %lld %lld %lld", &f32, &m, &d, &f) == 4) {
    const Plan a = plan_of(kForward, f32, m, f, d), b = plan_of(kInner, f32, m, f, d);
    const GradientsPlan g = plan_gradients(f32, m, d, f);
    std::printf("%d %d %d %d %d %d %d %d %d\n", a.shape, a.splits, b.shape, b.splits, (int)g.together, g.sum.shape,
                g.sum.splits, g.pair.shape, g.pair.splits);
  }
}
"""


def plans(sizes, folder):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src, exe = os.path.join(folder, "plan.cpp"), os.path.join(folder, "plan")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([cxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, src, "-o", exe], check=True)
    out = subprocess.run([exe], input="".join("%d %d %d %d\n" % s for s in sizes), capture_output=True, text=True,
                         check=True).stdout
    found = []
    for line in out.splitlines():
        v = [int(x) for x in line.split()]
        name = ["LMS"[v[i]] + str(v[i + 1]) for i in (0, 2, 5, 7)]
        found.append((name[0], name[1], (bool(v[4]), name[2], name[3])))
    assert len(found) == len(sizes)
    return found


def test_the_cases_take_what_they_name(tmp_path):
    found = plans([c[:4] for c in CASES], str(tmp_path))
    for case, plan in zip(CASES, found):
        assert case[4:] == plan, case


def test_the_cases_cover_the_instances():
    """Tile shapes, unsplit and split, of each product and type.  (A bfloat16 forward or inner
    product of larger tiles has no split that pays at any size looked at.)"""
    def kind(plan):
        return plan[0] + ("split" if plan != plan[0] + "1" else "")

    every = {"L", "Lsplit", "M", "Msplit", "S", "Ssplit"}
    for f32 in (False, True):
        mine = [c for c in CASES if c[0] == f32]
        for at in (4, 5):
            assert {kind(c[at]) for c in mine} == (every if f32 else {"L", "M", "S", "Ssplit"})
        apart = [c[6] for c in mine if not c[6][0]]
        assert {kind(p[1]) for p in apart} == every and {kind(p[2]) for p in apart} == every
        together = {(kind(p[1]), kind(p[2])) for _, *_, p in mine if p[0]}
        assert together == {(a + x, b + y) for a, b in ("SS", "LL", "LM") for x in ("", "split") for y in ("", "split")}
