"""The rules of csrc/softmax.h that shape the backward pass of softmax attention, compiled for the host, and which blocks they leave without work."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r'''
#include "softmax.h"
#include <stdio.h>
#include <stdlib.h>
using namespace aa;
int main(int argc, char** argv) {
  SoftmaxArgs a{};
  int v[9];
  for (int i = 0; i < 9; ++i) v[i] = atoi(argv[i + 1]);
  a.batch = v[0], a.heads_q = v[1], a.heads_k = v[2], a.tokens_q = v[3], a.tokens_k = v[4], a.d = v[5], a.causal = v[6], a.sequences = v[7];
  const SoftmaxBackPlan k = softmax_back_plan(a, v[8], true);
  printf("%d %d %d %d %lld\n", k.shared || (a.d > kTwoWidth && softmax_two_roundings(a, v[8])), softmax_step(v[8], softmax_width(a.d)), k.waves, k.splits, k.tiles);
}
'''


# batch, heads of queries and of keys, queries, keys, channels, causal: 16-bit calls with empty ranges
CAUSAL = [(1, 8, 8, 1024, 1024, 80, 1), (1, 8, 8, 1024, 1024, 128, 1), (1, 4, 4, 2048, 2048, 96, 1), (2, 4, 4, 1024, 1024, 128, 1),
          (1, 2, 1, 1500, 1500, 96, 1)]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """Of a call's sizes: whether two waves share the keys, queries of a tile, waves, ranges and tiles of keys."""
    d = tmp_path_factory.mktemp("plans")
    src, exe = d / "plans.cpp", d / "plans"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2312_08874_amd", "csrc"), str(src), "-o", str(exe)], check=True)

    def plan(B, Hq, Hk, nq, nk, d, causal=0, sequences=0, es=2):
        out = subprocess.run([str(exe)] + [str(x) for x in (B, Hq, Hk, nq, nk, d, causal, sequences, es)], check=True, capture_output=True, text=True)
        return dict(zip(("together", "step", "waves", "splits", "tiles"), (int(x) for x in out.stdout.split())))
    return plan


def empty_ranges(plan, B, Hq, Hk, nq, nk, d, causal):
    """Blocks of one head whose range of the queries' tiles is empty, two waves sharing their keys; else 0.  A causal tile of keys is seen by
    the tiles of queries from its first key's place on; a head's ranges take equal shares of them, rounded up."""
    if not plan["together"]:
        return 0
    empty = 0
    for tile in range(plan["tiles"]):
        first = max(0, 64 * tile - (nk - nq)) // plan["step"] if causal else 0
        tiles = Hq // Hk * max(0, -(-nq // plan["step"]) - first)
        each = -(-tiles // plan["splits"])
        empty += sum(split * each >= tiles for split in range(plan["splits"]))
    return empty
