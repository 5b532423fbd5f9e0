"""Host side of the layer norm: what is refused before anything is launched, workspaces, and the rule that shares a row out among
lanes (compiled from csrc/layer_norm.h)."""
import ctypes
import os
import subprocess

from paper_2312_08874_amd import binding
from paper_2312_08874_amd.binding import aa_layer_norm, aa_rows

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x100000      # never dereferenced: every call below fails before a launch


def desc(**kw):
    d = aa_layer_norm(rows=6, width=64, dtype=binding.AA_BF16, weight_dtype=binding.AA_F32, eps=1e-5)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def rows(p):
    p = p if isinstance(p, tuple) else (p, 0)
    return None if p[0] is None else ctypes.byref(aa_rows(*p))


def fwd(d=None, x=A, r=2 * A, w=3 * A, b=4 * A, y=5 * A, s=6 * A, saved=7 * A):
    d = desc() if d is None else d
    return binding.lib().agent_layer_norm_fwd(ctypes.byref(d) if d else None, rows(x), rows(r), w, b, rows(y), rows(s), saved, None)


def bwd(d=None, x=A, r=2 * A, dy=3 * A, saved=4 * A, w=5 * A, ds=6 * A, ws=7 * A, n=1 << 20, dx=8 * A, dw=20 * A, db=21 * A):
    d = desc() if d is None else d
    return binding.lib().agent_layer_norm_bwd(ctypes.byref(d), rows(x), rows(r), rows(dy), saved, w, rows(ds), ws, n, rows(dx), dw, db, None)


def test_refusals_of_the_descriptor():
    assert fwd(False) == -1
    for call in (fwd, bwd):
        assert call(desc(dtype=5)) == -3 and call(desc(weight_dtype=binding.AA_F16)) == -3 and call(desc(weight_dtype=9)) == -3
        for bad in (dict(rows=0), dict(width=0), dict(rows=-3), dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf"))):
            assert call(desc(**bad)) == -2, bad
        for bad in (dict(width=32769), dict(rows=(1 << 30) + 1)):
            assert call(desc(**bad)) == -7, bad


def test_refusals_of_the_forward_pass():
    assert fwd(x=None) == -1 and fwd(y=None) == -1
    for name in ("x", "r", "y", "s"):
        assert fwd(**{name: 9 * A + 1}) == -2, name
        assert fwd(**{name: (9 * A, 63)}) == -2, name
        assert fwd(**{name: (9 * A, 1 << 22)}) == -7, name
    assert fwd(w=3 * A + 2) == -2 and fwd(b=3 * A + 1) == -2 and fwd(saved=7 * A + 4) == -2
    assert fwd(s=5 * A) == -6 and fwd(y=A + 128) == -6 and fwd(y=(A, 80)) == -6 and fwd(s=2 * A + 64) == -6
    assert fwd(y=3 * A) == -6 and fwd(s=4 * A) == -6 and fwd(saved=A) == -6 and fwd(saved=5 * A) == -6 and fwd(saved=3 * A) == -6
    # columns of one buffer are apart, but where they are as wide as from one to the next
    assert fwd(y=(A + 100, 128), x=(A, 128)) == -6


def test_refusals_of_the_backward_pass():
    for name in ("x", "dy", "saved"):
        assert bwd(**{name: None}) == -1, name
    for name in ("x", "r", "dy", "ds", "dx"):
        assert bwd(**{name: 9 * A + 1}) == -2, name
    assert bwd(dw=20 * A + 2) == -2 and bwd(saved=4 * A + 4) == -2 and bwd(w=5 * A + 1) == -2
    need = binding.lib().agent_layer_norm_bwd_workspace_bytes(ctypes.byref(desc()))
    assert need == 2 * 64 * 4          # two sums of a column a block: 64 channels are four lanes, 64 rows a block
    assert binding.lib().agent_layer_norm_bwd_workspace_bytes(ctypes.byref(desc(rows=65))) == 2 * need
    assert bwd(ws=None) == -5 and bwd(ws=7 * A + 64) == -5 and bwd(n=need - 1) == -5
    assert bwd(dx=A + 64) == -6 and bwd(dx=5 * A) == -6 and bwd(dx=4 * A) == -6 and bwd(dw=A) == -6 and bwd(db=20 * A) == -6
    assert bwd(dw=5 * A) == -6 and bwd(ws=3 * A) == -6 and bwd(dx=7 * A) == -6 and bwd(db=7 * A) == -6
    assert binding.lib().agent_layer_norm_bwd_workspace_bytes(ctypes.byref(desc(rows=0))) == 0


RULES = r'''
#include "layer_norm.h"
#include <stdio.h>
using namespace aa;
int main() {
  for (int es = 2; es <= 4; es += 2)
    for (int back = 0; back < 2; ++back)
      for (int w = 1; w <= kNormWidth; w += w < 4200 ? 1 : 997) {
        const NormShape s = norm_shape(es, w, back);
        const int per = 16 / es;
        const bool pow2 = (s.lanes & (s.lanes - 1)) == 0;
        const bool known = s.pieces == 1 || s.pieces == 2 || s.pieces == 4 || (s.pieces == 8 && es == 4);
        const bool lanes = s.lanes <= 64 ? s.threads == 256 : s.lanes == s.threads && (s.lanes == 256 || s.lanes == 1024);
        const bool lds = s.lanes > 64 || !back || 8 * w * 4 <= 64 * 1024;
        if (!pow2 || !known || !lanes || !lds || s.lanes * s.pieces * per < w || s.lanes * s.pieces * per >= 4 * w + 64) printf("bad %d %d %d\n", es, back, w);
        for (int rows : {1, 5, 100000})
          if (norm_blocks(s, rows, back) < 1 || norm_blocks(s, rows, back) > (back ? kNormBlocks : 2048)) printf("blocks %d\n", w);
      }
  const NormShape last = norm_shape(2, kNormWidth, false);
  printf("%d %d\n", last.lanes, last.pieces);
}
'''


def test_rows_are_shared_out_among_lanes(tmp_path):
    src, exe = tmp_path / "rules.cpp", tmp_path / "rules"
    src.write_text("struct float2 { float x, y; };\n" + RULES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2312_08874_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout == "1024 4\n"
