"""Host side of the gated feed-forward block: what is refused before anything is launched, and the rule of its tiles."""
import ctypes
import os
import subprocess

import pytest

from paper_2312_08874_amd import binding
from paper_2312_08874_amd.binding import aa_ffn, aa_ffn_grads, aa_ffn_weights

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000000      # never dereferenced: every call below fails before a launch


def desc(**kw):
    d = dict(rows=12, width=64, hidden=96, dtype=binding.AA_BF16, activation=0, x_stride=0, y_stride=0, dx_stride=0)
    d.update(kw)
    return aa_ffn(*(d[n] for n, _ in aa_ffn._fields_))


OK = dict(w_gate=2 * A, w_up=3 * A, w_down=4 * A, b_gate=None, b_up=None, b_down=None)


def weights(**kw):
    w = dict(OK, **kw)
    return aa_ffn_weights(*(w[n] for n, _ in aa_ffn_weights._fields_))


def fwd(d=None, x=A, w=None, saved=None, ws=6 * A, size=1 << 26, y=5 * A):
    d, w = desc() if d is None else d, weights() if w is None else w
    return binding.lib().agent_gated_ffn_fwd(ctypes.byref(d), x, ctypes.byref(w), saved, ws, size, y, None)


def bwd(d=None, x=A, w=None, saved=8 * A, dy=9 * A, ws=6 * A, size=1 << 26, dx=5 * A, **grads):
    d, w, g = desc() if d is None else d, weights() if w is None else w, aa_ffn_grads(**grads)
    return binding.lib().agent_gated_ffn_bwd(ctypes.byref(d), x, ctypes.byref(w), saved, dy, ws, size, dx, ctypes.byref(g), None)


def test_refusals_of_the_descriptor():
    assert binding.lib().agent_gated_ffn_fwd(None, A, ctypes.byref(weights()), None, 6 * A, 1 << 26, 5 * A, None) == -1
    sizes = (binding.lib().agent_gated_ffn_workspace_bytes, binding.lib().agent_gated_ffn_saved_bytes,
             binding.lib().agent_gated_ffn_bwd_workspace_bytes)
    for status, cases in ((-3, [dict(dtype=4)]),
                          (-2, [dict(rows=0), dict(width=0), dict(hidden=-1), dict(activation=5), dict(activation=-1),
                                dict(x_stride=63), dict(y_stride=-64), dict(dx_stride=1)]),
                          (-7, [dict(width=(1 << 20) + 1), dict(hidden=1 << 21), dict(x_stride=1 << 22),
                                dict(rows=1 << 30, hidden=1 << 12)])):
        for kw in cases:
            assert fwd(desc(**kw)) == status and bwd(desc(**kw)) == status, kw
            assert all(f(ctypes.byref(desc(**kw))) == 0 for f in sizes)
    assert all(f(ctypes.byref(desc())) % 256 == 0 and f(ctypes.byref(desc())) > 0 for f in sizes)


def test_refusals_of_the_forward_pass():
    assert fwd(x=None) == -1 and fwd(y=None) == -1
    for name in ("w_gate", "w_up", "w_down"):
        assert fwd(w=weights(**{name: None})) == -1
    assert binding.lib().agent_gated_ffn_fwd(ctypes.byref(desc()), A, None, None, 6 * A, 1 << 26, 5 * A, None) == -1
    need = binding.lib().agent_gated_ffn_workspace_bytes(ctypes.byref(desc()))
    assert fwd(ws=None) == -5 and fwd(ws=6 * A + 128) == -5 and fwd(size=need - 1) == -5
    assert fwd(saved=8 * A + 16) == -5
    assert fwd(x=A + 1) == -2 and fwd(w=weights(b_up=7 * A + 1)) == -2 and fwd(y=5 * A + 1) == -2
    assert fwd(y=A + 64) == -6 and fwd(y=2 * A) == -6 and fwd(y=6 * A + 64) == -6
    assert fwd(ws=A, size=need) == -6 and fwd(saved=6 * A + 256) == -6 and fwd(saved=2 * A) == -6
    assert fwd(w=weights(b_down=5 * A + 32)) == -6
    assert fwd(desc(x_stride=1000), y=A + 11 * 2000) == -6                                # inside x's last row


def test_refusals_of_the_backward_pass():
    for kw in (dict(x=None), dict(saved=None), dict(dy=None), dict(w=weights(w_up=None))):
        assert bwd(**kw) == -1
    need = binding.lib().agent_gated_ffn_bwd_workspace_bytes(ctypes.byref(desc()))
    assert bwd(ws=None) == -5 and bwd(ws=6 * A + 1) == -5 and bwd(size=need - 1) == -5 and bwd(saved=8 * A + 16) == -5
    assert bwd(dx=9 * A) == -6 and bwd(dx=A) == -6 and bwd(dx=8 * A + 512) == -6
    assert bwd(dw_gate=2 * A) == -6 and bwd(dw_gate=5 * A) == -6 and bwd(dw_gate=7 * A, dw_up=7 * A + 64) == -6
    assert bwd(db_down=9 * A + 2) == -6 and bwd(db_gate=7 * A + 1) == -2


def test_struct_layouts():
    assert ctypes.sizeof(aa_ffn) == 48 and aa_ffn.x_stride.offset == 24
    assert ctypes.sizeof(aa_ffn_weights) == 48 and ctypes.sizeof(aa_ffn_grads) == 48


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    at = tmp_path_factory.mktemp("rule")
    (at / "r.cpp").write_text('''#include "%s/paper_2312_08874_amd/csrc/ffn.h"
extern "C" void tile(long long M, long long N, long long M2, long long N2, int steps, int es, int split, int gated, int* out) {
  const aa::FfnTile t = aa::ffn_tile(M, N, M2, N2, steps, es, split, gated, 256);
  out[0] = t.rows, out[1] = t.cols, out[2] = t.full, out[3] = t.parts, out[4] = t.each;
}
extern "C" int pitch(int hidden) { return aa::ffn_pitch(hidden); }
extern "C" void place(unsigned at, unsigned m, unsigned n, int* out) { aa::ffn_place(at, m, n, out[0], out[1]); }
extern "C" unsigned run(unsigned L, unsigned count) { return aa::ffn_run(L, count); }
''' % ROOT)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-o", str(at / "r.so"), str(at / "r.cpp")], check=True)
    lib = ctypes.CDLL(str(at / "r.so"))
    lib.tile.argtypes = [ctypes.c_longlong] * 4 + [ctypes.c_int] * 4 + [ctypes.c_void_p]
    return lib


def tile(rule, M, N, steps, es, split, gated, M2=0, N2=0):
    out = (ctypes.c_int * 5)()
    rule.tile(M, N, M2, N2, steps, es, int(split), int(gated), out)
    return tuple(out)


def test_tiles_and_parts(rule):
    assert rule.pitch(1) == 64 and rule.pitch(64) == 64 and rule.pitch(1365) == 1408
    for M in (1, 60, 196, 4096, 100000):
        for N in (8, 512, 5504):
            for steps in (1, 3, 8, 40, 1000):
                for es in (2, 4):
                    for split, gated in ((False, True), (True, False)):
                        for M2 in (0, 300) if split else (0,):
                            rows, cols, full, parts, each = tile(rule, M, N, steps, es, split, gated, M2, 700)
                            assert (rows, cols) in (((256, 256), (256, 128), (128, 128), (64, 64)) if es == 2 else ((128, 128), (64, 64)))
                            of = cols // 2 if gated else cols
                            tiles = -(-M // rows) * -(-N // of) + (-(-M2 // rows) * -(-700 // of))
                            assert parts >= 1 and (split or parts == 1) and 0 <= full <= tiles
                            if parts > 1:      # every part has steps of its own, and the tail's launch fits its grid
                                assert full < tiles and tiles - full < 65536
                                assert (parts - 1) * each < steps <= parts * each
                            else:
                                assert full == tiles
    assert tile(rule, 8192, 5504, 32, 2, False, True)[:2] == (256, 256)
    assert tile(rule, 1, 64, 8, 2, True, False)[0] == 64


def test_every_tile_has_one_block(rule):
    for m, n in ((1, 1), (7, 3), (8, 8), (9, 5), (23, 17), (64, 2)):
        seen, out = set(), (ctypes.c_int * 2)()
        for at in range(m * n):
            rule.place(at, m, n, out)
            assert 0 <= out[0] < m and 0 <= out[1] < n
            seen.add(tuple(out))
        assert len(seen) == m * n
    for count in (1, 7, 8, 9, 255, 256, 300):
        got = [rule.run(L, count) for L in range((count + 7) // 8 * 8)]
        assert sorted(x for x in got if x < count) == list(range(count))
