"""The layer norm's kernels are compiled for what its rule comes to over all widths, and for nothing else (csrc/layer_norm.h)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r'''
struct float2 {
  float x, y;
};
#include "layer_norm.h"
#include <stdio.h>
#include <set>
#include <tuple>
using namespace aa;
int main() {
  for (const int es : {2, 4})
    for (const bool back : {false, true}) {
      std::set<std::tuple<int, bool, int>> reached, compiled;
      for (int w = 1; w <= kNormWidth; ++w) {
        const NormShape s = norm_shape(es, w, back);
        if (s.lanes * s.pieces * (16 / es) < w) return printf("width %d is not covered\n", w), 1;
        reached.insert({s.threads, s.lanes >= 256, s.pieces});
      }
      for (int pieces = 1; pieces <= (es == 4 ? 8 : 4); pieces *= 2)
        for (const auto& k : {std::make_pair(256, false), std::make_pair(256, true), std::make_pair(1024, true)})
          if (norm_takes(es, k.first, k.second, pieces, back)) compiled.insert({k.first, k.second, pieces});
      for (const auto& [threads, block, pieces] : reached)
        if (!compiled.count({threads, block, pieces})) printf("es %d back %d: %d %d %d is reached and not compiled\n", es, back, threads, block, pieces);
      for (const auto& [threads, block, pieces] : compiled)
        if (!reached.count({threads, block, pieces})) printf("es %d back %d: %d %d %d is compiled and not reached\n", es, back, threads, block, pieces);
    }
}
'''


def test_kernels_are_those_that_widths_lead_to(tmp_path):
    src, exe = tmp_path / "shapes.cpp", tmp_path / "shapes"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2312_08874_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "", r.stdout
