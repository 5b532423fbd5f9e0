"""Host side of softmax attention: what is refused before anything is launched, workspaces, and the rules that shape the kernels
(compiled from csrc/softmax.h)."""
import ctypes
import os
import subprocess

import pytest

from paper_2312_08874_amd import binding
from paper_2312_08874_amd.binding import aa_softmax_attn, aa_view

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x100000      # never dereferenced: every call below fails before a launch


def desc(**kw):
    d = aa_softmax_attn(batch=2, heads_q=4, heads_k=2, tokens_q=12, tokens_k=20, d=32, dtype=binding.AA_BF16)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def view(p, strides=(0, 0, 0)):
    return None if p is None else ctypes.byref(aa_view(p, *strides))


def fwd(d=None, q=A, k=2 * A, v=3 * A, out=4 * A, saved=None, ws=None, n=0, st=((0, 0, 0),) * 4):
    return binding.lib().agent_softmax_attn_fwd(None if d is None else ctypes.byref(d), view(q, st[0]), view(k, st[1]), view(v, st[2]),
                                                ws, n, view(out, st[3]), saved, None)


def bwd(d=None, q=A, k=2 * A, v=3 * A, out=4 * A, saved=5 * A, dout=6 * A, ws=7 * A, n=1 << 30, dq=1 << 31, dk=(1 << 31) + A,
        dv=(1 << 31) + 2 * A):
    d = desc() if d is None else d
    return binding.lib().agent_softmax_attn_bwd(ctypes.byref(d), view(q), view(k), view(v), view(out), saved, view(dout), ws, n, view(dq),
                                                view(dk), view(dv), None)


def need(d, views=(A, 2 * A, 3 * A), back=False):
    L = binding.lib()
    if back:
        return L.agent_softmax_attn_bwd_workspace_bytes(ctypes.byref(d), *(view(p) for p in views), view(6 * A))
    return L.agent_softmax_attn_workspace_bytes(ctypes.byref(d), *(view(p) for p in views))


def test_refusals_of_the_descriptor():
    assert fwd(None) == -1
    assert fwd(desc(dtype=9)) == -3
    for bad in (dict(batch=0), dict(heads_q=0), dict(heads_k=0), dict(heads_k=-2), dict(tokens_q=0), dict(tokens_k=-1), dict(d=0),
                dict(heads_k=3), dict(sequences=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38),
                dict(sequences=2, starts_q=A, starts_k=A),                                    # a batch of two, packed
                dict(starts_q=A), dict(starts_k=A),                                           # starts of nothing
                dict(batch=1, sequences=2, starts_q=A, starts_k=A, lengths_q=A), dict(lengths_k=A + 2), dict(lengths_q=A + 1)):
        assert fwd(desc(**bad)) == -2, bad
    assert fwd(desc(batch=1, sequences=2, starts_q=A)) == -1
    assert fwd(desc(batch=1, sequences=2, starts_k=A)) == -1
    for bad in (dict(d=257), dict(heads_q=131072), dict(tokens_q=(1 << 30) + 1), dict(sequences=(1 << 28) + 1, batch=1, starts_q=A, starts_k=A),
                dict(batch=1 << 20, tokens_k=1 << 20), dict(batch=1 << 28, heads_q=16, heads_k=16, tokens_q=1, tokens_k=1)):
        assert fwd(desc(**bad)) == -7, bad
        assert bwd(desc(**bad)) == -7, bad


def test_refusals_of_tensors():
    for name in ("q", "k", "v", "out"):
        assert fwd(desc(), **{name: None}) == -1
        assert fwd(desc(), **{name: 9 * A + 1}) == -2
    dense = (0, 0, 0)
    assert fwd(desc(), st=(dense, dense, dense, (12 * 128, 16, 128))) == -2        # heads of the result overlap
    assert fwd(desc(), st=(dense, dense, dense, (0, 32, 128))) == -2               # its sequences coincide
    assert fwd(desc(), st=((-1, 32, 128), dense, dense, dense)) == -2
    assert fwd(desc(), st=((1 << 41, 32, 128), dense, dense, dense)) == -7
    assert fwd(desc(), out=A) == -6                                                # over the queries
    assert fwd(desc(), out=2 * A + 64) == -6
    assert fwd(desc(), saved=4 * A + 256) == -6
    assert fwd(desc(), saved=A + 128) == -5                                        # not aligned
    assert fwd(desc(batch=1, sequences=1, starts_q=4 * A, starts_k=9 * A)) == -6   # starts inside the result
    assert fwd(desc(lengths_k=4 * A + 8)) == -6
    # slices of one projection [2,12,8,32]: the result in a slice of its own is apart, one row further it is not
    f = (12 * 256, 32, 256)
    d = desc(tokens_k=12)
    bad = fwd(d, A, A + 4 * 64, A + 6 * 64, A + 2 * 64, st=(f, f, f, f))
    assert bad == -6


def test_refusals_of_the_backward_pass():
    for name in ("q", "k", "v", "out", "saved", "dout", "dq", "dk", "dv"):
        assert bwd(**{name: None}) == -1, name
    for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        assert bwd(**{name: 9 * A + 1}) == -2, name
    assert bwd(ws=None) == -5 and bwd(ws=7 * A + 128) == -5 and bwd(saved=5 * A + 8) == -5
    assert bwd(n=need(desc(), back=True) - 1) == -5
    assert bwd(dq=A) == -6 and bwd(dq=6 * A) == -6 and bwd(dk=2 * A) == -6 and bwd(dv=(1 << 31) + A) == -6 and bwd(dk=7 * A) == -6
    assert bwd(dv=5 * A) == -6


def test_workspaces():
    aligned = desc()
    assert need(aligned) == 0                                          # whole pieces, read where they lie
    assert need(aligned, views=(A, 2 * A + 2, 3 * A)) == 2 * 2 * 20 * 32 * 2      # one tensor off its pieces is copied
    assert need(aligned, views=(None, None, None)) > need(aligned, views=(A, 2 * A + 2, 3 * A))
    odd = desc(d=33)
    rows = (2 * 4 * 12, 2 * 2 * 20, 2 * 2 * 20)                        # 33 channels lie 40 apart, pieces of 16 bytes
    assert need(odd) == sum(-(-r * 40 * 2 // 256) * 256 for r in rows)
    assert fwd(odd) == -5 and fwd(odd, ws=8 * A, n=need(odd) - 1) == -5
    # single tokens over long keys leave parts: fp32 accumulators and two statistics a row and range
    long = desc(tokens_q=1, tokens_k=65536)
    parts = need(long)
    assert parts > 0 and parts % 256 == 0
    assert fwd(long) == -5
    assert need(desc(d=300)) == 0 and need(desc(d=300), back=True) == 0
    rows = 2 * 4 * 12
    assert need(desc(), back=True) == 8 * rows                         # two statistics a query
    assert need(desc(dtype=binding.AA_F16), back=True) == 4096 + 8 * rows      # and the blocks' largest rows of dout and v
    L = binding.lib()
    assert L.agent_softmax_attn_saved_bytes(ctypes.byref(desc())) == 512 + 2 * 4 * 12 * 32 * 2
    assert L.agent_softmax_attn_saved_bytes(ctypes.byref(desc(dtype=binding.AA_F32))) == 512
    assert L.agent_softmax_attn_saved_bytes(ctypes.byref(desc(d=0))) == 0


RULES = r'''
#include "softmax.h"
#include <stdio.h>
#include <stdlib.h>
using namespace aa;
int main(int argc, char** argv) {
  SoftmaxArgs a{};
  int v[9];
  for (int i = 0; i < 9; ++i) v[i] = atoi(argv[i + 1]);
  a.batch = v[0], a.heads_q = v[1], a.heads_k = v[2], a.tokens_q = v[3], a.tokens_k = v[4], a.d = v[5], a.causal = v[6], a.sequences = v[7];
  const SoftmaxPlan p = softmax_plan(a, v[8]);
  const SoftmaxBackPlan q = softmax_back_plan(a, v[8], false), k = softmax_back_plan(a, v[8], true);
  printf("%d %d %d %d %d %d %d %d %lld %d %d %lld %d %d %lld\n", p.shared, q.shared, k.shared, p.columns, p.waves, p.pack, p.tile_tokens, p.splits, p.tiles, q.waves, q.splits, q.tiles,
         k.waves, k.splits, k.tiles);
}
'''


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    src, exe = d / "rules.cpp", d / "rules"
    src.write_text(RULES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2312_08874_amd", "csrc"), str(src), "-o", str(exe)], check=True)

    def plan(B, Hq, Hk, nq, nk, d, causal=0, sequences=0, es=2):
        out = subprocess.run([str(exe)] + [str(x) for x in (B, Hq, Hk, nq, nk, d, causal, sequences, es)], check=True, capture_output=True, text=True)
        names = ("shared", "dq_shared", "dkv_shared", "columns", "waves", "pack", "tile_tokens", "splits", "tiles", "dq_waves", "dq_splits", "dq_tiles", "dkv_waves", "dkv_splits", "dkv_tiles")
        return dict(zip(names, (int(x) for x in out.stdout.split())))
    return plan


def test_which_kernel_takes_what(rules):
    one = rules(8, 16, 4, 1, 65536, 128, 1)
    assert one["columns"] and one["pack"] == 4 and one["tile_tokens"] == 8 and one["splits"] == 16 and one["tiles"] == 1
    assert not rules(64, 3, 3, 196, 196, 64)["columns"]
    big = rules(1, 8, 8, 16384, 16384, 64)
    assert not big["columns"] and big["waves"] == 8 and big["tiles"] == 64 and big["dkv_waves"] == 4 and big["dq_splits"] == 1
    assert rules(2048, 12, 12, 49, 49, 32)["waves"] == 2                  # half of 128 rows would be empty
    assert rules(1, 2, 2, 64, 20000, 64)["columns"]                       # few blocks, long keys
    assert not rules(1, 2, 2, 64, 300, 64)["columns"]
    few = rules(2, 8, 8, 1500, 1500, 64)                                  # 384 blocks of 64 rows, whose keys two waves share
    assert few["waves"] == few["dq_waves"] == few["dkv_waves"] == 2 and few["shared"] and few["dq_shared"] and few["dkv_shared"]
    assert not rules(2, 8, 8, 1500, 1500, 64, es=4)["shared"] and not big["shared"] and not one["shared"]
    # every token has a tile, whatever the lengths on the device are
    for case in ((1, 4, 2, 1000, 1300, 64, 0, 7), (1, 4, 4, 70, 900, 64, 1, 70), (1, 8, 1, 33, 5, 128, 0, 1), (1, 1, 1, 1, 1, 8, 0, 1)):
        p = rules(*case)
        assert p["tiles"] == case[3] // p["tile_tokens"] + case[7]
        assert p["dkv_tiles"] == case[4] // (32 * p["dkv_waves"]) + case[7]
    assert rules(1, 2, 2, 200, 200, 128)["dkv_waves"] == 2 == rules(1, 2, 2, 200, 200, 128)["dq_waves"]      # two roundings: two waves
    for hq, hk in ((1, 1), (6, 2), (5, 1), (12, 3), (64, 1), (7, 7)):
        p = rules(3, hq, hk, 1, 5000, 64)
        assert (hq // hk) % p["pack"] == 0 and 1 <= p["pack"] <= 32 and p["tile_tokens"] == 32 // p["pack"]
    for es in (2, 4):
        for n in (1, 17, 500, 4000, 30000):
            p = rules(1, 2, 1, n, n, 64, 1, 0, es)
            assert 1 <= p["splits"] <= 128 and 1 <= p["dq_splits"] <= 128 and 1 <= p["dkv_splits"] <= 128
            assert p["tiles"] * p["tile_tokens"] >= n and p["dq_tiles"] * 32 * p["dq_waves"] >= n
