"""The tiles and splits of the products grouped by expert: a host rule, compiled here with
the C++ compiler (no GPU)."""
import os
import shutil
import subprocess

import pytest

from _expert_cases import CASES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "isoloco_experts_plan.h"
#include <stdio.h>
using namespace isoloco;
int main() {
  const long sizes[] = {1, 7, 64, 65, 300, 612, 1408, 2048, 5632, 70000}, many[] = {1, 5, 64, 1024};
  long n = 0;
  for (long rows : {0L, 1L, 63L, 700L, 4096L, 131072L, 2147483647L})
    for (long experts : many)
      for (long dim : sizes)
        for (long cols : sizes)
          for (int f32 = 0; f32 < 2; ++f32) {
            const ExpertPlan o = expert_plan(kOut, f32, rows, experts, 0, cols, dim);
            const ExpertGradients g = expert_plan_gradients(f32, rows, experts, dim, cols);
            for (const ExpertPlan& p : {o, g.dx, g.dw}) {
              if (p.shape < 0 || p.shape >= kShapes || p.splits < 1 || p.splits > kMaxSplits || !(p.us > 0)) return 1;
            }
            // every split has slabs to take, and dw has no 192 x 256 tiles
            const long slabs_out = (dim + 63) / 64 * (f32 ? 6 : 1), slabs_dx = (cols + 63) / 64 * (f32 ? 6 : 1);
            if (o.splits > 1 && o.splits * 4 > slabs_out) return 2;
            if (g.dx.splits > 1 && g.dx.splits * 4 > slabs_dx) return 3;
            if (g.dw.shape == kMiddle) return 4;
            // one launch has one tile shape
            if (g.together && g.dx.shape != g.dw.shape) return 5;
            const size_t wx = expert_partial_bytes(g.dx, kDx, rows, experts, 0, dim);
            if (wx != (g.dx.splits > 1 ? (size_t)g.dx.splits * rows * ((dim + 63) / 64 * 64) * 4 : 0)) return 6;
            ++n;
          }
  printf("%ld\n", n);
  return 0;
}
"""


def test_plans(tmp_path):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2607_03011_amd", "csrc"),
                    str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, "case %d" % out.returncode
    assert int(out.stdout) == 7 * 4 * 100 * 2


def test_cases_take_what_they_say(tmp_path):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    calls = "\n".join("  show(%d, %d, %d, %d, %d);" % (kind == "f32", e, r, d, c) for kind, e, r, d, c, _ in CASES)
    src, exe = tmp_path / "cases.cpp", tmp_path / "cases"
    src.write_text(r"""
#include "isoloco_experts_plan.h"
#include <stdio.h>
using namespace isoloco;
static void one(const ExpertPlan& p) { printf("%c%d", "LMS"[p.shape], p.splits); }
static void show(bool f32, long experts, long rows, long dim, long cols) {
  const ExpertGradients g = expert_plan_gradients(f32, rows, experts, dim, cols);
  one(expert_plan(kOut, f32, rows, experts, 0, cols, dim));
  printf(" ");
  one(g.dx);
  printf(g.together ? "+" : " ");
  one(g.dw);
  printf("\n");
}
int main() {
""" + calls + "\n}\n")
    subprocess.run([cxx, "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_03011_amd", "csrc"), str(src), "-o", str(exe)],
                   check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()
    seen = set()
    for line, (kind, _, _, _, _, plan) in zip(got, CASES, strict=True):
        if plan.startswith("few"):
            line = "few " + line.split(" ", 1)[1]
        assert line == plan
        out, back = plan.split(" ", 1)
        dx, dw = back.replace("+", " ").split()
        seen |= {(kind, "out", out[0]), (kind, "dx", dx[0]), (kind, "dw", dw[0])}
        if "+" in back:
            seen.add((kind, "both", dx[0]))
    for kind in ("bf16", "f32"):
        for tile in "LMS":
            assert {(kind, "out", tile), (kind, "dx", tile)} <= seen
        for tile in "LS":
            assert {(kind, "dw", tile), (kind, "both", tile)} <= seen
