"""Host side of the rotary positions and the norms of queries and keys: what is refused before anything is launched, and
the rules that shape the kernels (compiled from csrc/rotary.h)."""
import ctypes
import os
import subprocess

import pytest

from paper_2312_08874_amd import binding
from paper_2312_08874_amd.binding import aa_qk_norm, aa_rotary, aa_view

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, FAR = 0x100000, 1 << 40      # never dereferenced: every call below fails before a launch


def desc(**kw):
    freq = (ctypes.c_double * 128)(*([1.0] * 128))
    d = aa_rotary(batch=2, tokens=12, heads_q=3, heads_k=3, d=32, dtype=binding.AA_BF16, pairing=1, axes=2,
                  freq=ctypes.addressof(freq))
    d.pairs[:2], d.grid[:2] = (8, 8), (3, 4)
    d.keep = freq
    for k, v in kw.items():
        if k in ("pairs", "grid"):
            for i, x in enumerate(v):
                getattr(d, k)[i] = x
        else:
            setattr(d, k, v)
    return d


def views(q=A, k=2 * A, qo=3 * A, ko=4 * A, strides=None):
    st = strides or ((0, 0, 0),) * 4
    return [None if p is None else ctypes.byref(aa_view(p, *s)) for p, s in zip((q, k, qo, ko), st)]


def rope(d=None, **kw):
    return binding.lib().agent_rope_fwd(None if d is None else ctypes.byref(d), *views(**kw), None)


def test_refusals_of_the_descriptor():
    assert rope(None) == -1
    assert rope(desc(dtype=7)) == -3
    for bad in (dict(batch=0), dict(tokens=0), dict(heads_q=0), dict(heads_k=-1), dict(d=0), dict(axes=-1), dict(axes=5),
                dict(axes=0), dict(pairing=3), dict(pairing=-1), dict(pairs=(0, 8)), dict(pairs=(9, 8)), dict(pairs=(-1, 3)),
                dict(pairs=(2 ** 31 - 1, 8)), dict(grid=(3, 5)), dict(grid=(12, 0)), dict(grid=(-3, -4)),
                dict(grid=(65536, 65536)), dict(positions=A), dict(positions=A + 2, grid=(0, 0))):
        assert rope(desc(**bad)) == -2, bad
    for bad in (dict(d=258), dict(batch=1 << 20, tokens=1 << 20, grid=(1 << 10, 1 << 10)), dict(heads_q=70000)):
        assert rope(desc(**bad)) == -7, bad
    assert rope(desc(freq=None)) == -1
    assert rope(desc(grid=(0, 0))) == -1                     # neither a grid nor positions
    d = desc()
    d.keep[5] = float("nan")
    assert rope(d) == -2


def test_refusals_of_tensors():
    for name in ("q", "k", "qo", "ko"):
        assert rope(desc(), **{name: None}) == -1
        assert rope(desc(), **{name: 9 * A + 1}) == -2                                     # not an element's address
    dense, tight = (0, 0, 0), (12 * 96, 16, 96)
    assert rope(desc(), strides=(dense, dense, tight, dense)) == -2                        # heads of a result overlap
    assert rope(desc(), strides=(dense, dense, (0, 32, 96), dense)) == -2                  # sequences of a result coincide
    assert rope(desc(), strides=((-1, 32, 96), dense, dense, dense)) == -2
    assert rope(desc(), strides=((1 << 41, 32, 96), dense, dense, dense)) == -7
    assert rope(desc(), ko=3 * A + 64) == -6                                               # results overlap
    assert rope(desc(), qo=2 * A) == -6                                                    # a result is the other's input
    assert rope(desc(), qo=A + 64) == -6                                                   # shifted against its own input
    st = (12 * 96, 32, 96)
    assert rope(desc(), qo=A, strides=(dense, dense, st, dense)) == -6                     # in place with other strides
    # slices of one projection [2,12,3,3,32], one of them written over its neighbour's first head
    f = (12 * 288, 32, 288)
    assert rope(desc(), q=A, k=A + 192, qo=A + 128, ko=4 * A, strides=(f, f, f, dense)) == -6
    # positions inside a result
    assert rope(desc(grid=(0, 0), positions=3 * A + 64)) == -6


def test_refusals_of_the_norm():
    L, ok = binding.lib(), aa_qk_norm(5 * A, 6 * A, 0, 1e-6)

    def fwd(d, n, **kw):
        return L.agent_qk_norm_fwd(ctypes.byref(d), None if n is None else ctypes.byref(n), *views(**kw), None)
    assert fwd(desc(), None) == -1
    for eps in (-1.0, float("nan"), float("inf")):
        assert fwd(desc(), aa_qk_norm(5 * A, 6 * A, 0, eps)) == -2
    assert fwd(desc(), aa_qk_norm(5 * A + 2, 6 * A, 0, 0.0)) == -2
    assert fwd(desc(), aa_qk_norm(3 * A + 8, None, 0, 0.0)) == -6                          # weights inside a result
    assert fwd(desc(d=300), ok) == -7

    def bwd(d=None, n=ok, ws=7 * A, size=FAR, dw=(8 * A, 9 * A), q=A, dq=FAR, dk=2 * FAR):
        d = desc() if d is None else d
        v = [ctypes.byref(aa_view(p, 0, 0, 0)) for p in (q, 2 * A, 3 * A, 4 * A)]
        out = [ctypes.byref(aa_view(p, 0, 0, 0)) for p in (dq, dk)]
        return L.agent_qk_norm_bwd(ctypes.byref(d), ctypes.byref(n), *v, ws, size, *out, *dw, None)
    need = L.agent_qk_norm_bwd_workspace_bytes(ctypes.byref(desc()), ctypes.byref(ok))
    assert need > 0 and need % 256 == 0
    assert L.agent_qk_norm_bwd_workspace_bytes(ctypes.byref(desc(tokens=11)), ctypes.byref(ok)) == 0
    assert bwd(ws=None) == -5 and bwd(ws=7 * A + 8) == -5 and bwd(size=need - 1) == -5
    assert bwd(ws=A, size=need) == -6 and bwd(ws=FAR + 256, size=need) == -6
    assert bwd(size=need, dw=(8 * A + 2, None)) == -2
    assert bwd(size=need, dw=(5 * A, None)) == -6 and bwd(size=need, dw=(8 * A, 8 * A + 64)) == -6
    assert bwd(size=need, dw=(A + 64, None)) == -6 and bwd(size=need, dw=(7 * A, None)) == -6
    assert bwd(dq=4 * A, dw=(None, None)) == -6                                            # dq over dk_out


def test_the_binding_refuses():
    torch = pytest.importorskip("torch")
    with pytest.raises(AssertionError):
        binding.Rope((8, 8))
    with pytest.raises(AssertionError):
        binding.Rope((8, 8), grid=(3,))
    with pytest.raises(AssertionError):
        binding.Rope((8, 0), grid=(3, 4))
    with pytest.raises(AssertionError):
        binding.Rope((8,), grid=(3,), freqs=[1.0])
    with pytest.raises(AssertionError):
        binding.Rope((8,), positions=torch.zeros(3, 1))                                    # host memory
    with pytest.raises(AssertionError):
        binding.Rope((8,), grid=(3,), pairing="other")
    assert binding.rope_frequencies((2, 1), 100.0) == [1.0, 0.1, 1.0]
    assert binding.rope_frequencies((1, 1), 100.0, shared=True) == [1.0, 0.1]


def test_struct_layouts():
    assert ctypes.sizeof(aa_view) == 32 and ctypes.sizeof(aa_rotary) == 88 and ctypes.sizeof(aa_qk_norm) == 24
    assert aa_rotary.freq.offset == 64


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    at = tmp_path_factory.mktemp("rules")
    src = at / "r.cpp"
    src.write_text('''#include "%s/paper_2312_08874_amd/csrc/rotary.h"
extern "C" void shape(int es, int d, int pairing, int axes, const int* first, unsigned long long align, int* out) {
  const aa::RotaryShape s = aa::rotary_shape(es, d, pairing, axes, first, align);
  out[0] = s.ve, out[1] = s.lanes, out[2] = s.duos;
}
extern "C" void plan(long long rows, int heads_q, int heads_k, int lanes, int backward, int one_head, int* out) {
  const aa::RotaryPlan p = aa::rotary_plan({1, lanes, 1}, rows, heads_q, heads_k, backward, one_head);
  out[0] = p.shift, out[1] = p.across, out[2] = p.chunk, out[3] = p.chunks[0], out[4] = p.chunks[1], out[5] = p.tiles, out[6] = p.blocks;
}
''' % ROOT)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-o", str(at / "r.so"), str(src)], check=True)
    return ctypes.CDLL(str(at / "r.so"))


def shape(rules, es, d, pairing, pairs, align=0):
    first = [0]
    for p in pairs:
        first.append(first[-1] + p)
    out = (ctypes.c_int * 3)()
    rules.shape(es, d, pairing, len(pairs), (ctypes.c_int * 5)(*(first + [first[-1]] * (5 - len(first)))),
                ctypes.c_ulonglong(align), out)
    return tuple(out)


def test_shapes_of_the_kernels(rules):
    assert shape(rules, 2, 64, 1, (16, 16)) == (8, 4, 1)
    assert shape(rules, 2, 40, 0, (10, 10)) == (8, 4, 1)
    assert shape(rules, 2, 40, 1, (10, 10)) == (4, 8, 1)            # halves 20 channels apart
    assert shape(rules, 2, 128, 1, (22, 21, 21)) == (8, 8, 1)       # halves 64 apart
    assert shape(rules, 2, 128, 2, (22, 21, 21)) == (1, 16, 4)
    assert shape(rules, 4, 48, 2, (12, 12)) == (4, 8, 1)
    assert shape(rules, 4, 256, 0, (128,)) == (4, 32, 1)
    assert shape(rules, 2, 64, 1, (16, 16), align=2) == (1, 8, 4)
    assert shape(rules, 2, 64, 1, (16, 16), align=12) == (2, 8, 2)
    assert shape(rules, 2, 1, 0, ()) == (1, 1, 4)
    for es in (2, 4):      # every width is covered by its lanes, and no load is wider than what divides everything
        for d in range(1, 257):
            for align in (0, 2, 4, 8, 16):
                if align % es:
                    continue
                ve, lanes, duos = shape(rules, es, d, 0, (), align)
                assert lanes <= 64 and lanes * duos * 2 * ve >= d and d % ve == 0 and align % (ve * es) == 0


def test_launches_cover_every_row(rules):
    rules.plan.argtypes = [ctypes.c_longlong] + [ctypes.c_int] * 5 + [ctypes.c_void_p]

    def plan(*args):
        out = (ctypes.c_int * 7)()
        rules.plan(*args, out)
        return tuple(out)
    assert plan(1, 8, 8, 4, 0, 0)[:5] == (2, 4, 1, 4, 0)            # one token: every wave a head of its own
    assert plan(1 << 20, 16, 4, 8, 0, 0)[:5] == (3, 4, 5, 1, 0)     # many: a block takes all heads of its tokens
    for rows in (1, 2, 63, 1000, 12544, 70001, 1 << 22, (1 << 31) - 1):
        for heads in ((1, 0), (1, 1), (2, 1), (3, 3), (16, 4), (40, 0), (7, 300)):
            for lanes in (1, 4, 64):
                for backward, one_head in ((0, 0), (1, 0), (1, 1)):
                    shift, across, chunk, cq, ck, tiles, blocks = plan(rows, *heads, lanes, backward, one_head)
                    tokens = 4 // across * (64 // lanes)
                    assert 1 << shift == lanes and across in ((1, 2) if backward else (1, 2, 4)) and chunk >= 1 and (chunk == 1 or not one_head)
                    assert (tiles - 1) * tokens < rows <= tiles * tokens and 1 <= blocks <= tiles
                    share = across * chunk
                    for c, n in ((cq, heads[0]), (ck, heads[1])) if backward else ((cq, sum(heads)), (ck, 0)):
                        assert (c - 1) * share < n <= c * share
                    if backward:      # the sums' workspace
                        assert blocks * (1 if one_head else max(cq, ck)) <= max(1024, sum(heads))
                    else:
                        assert blocks == tiles
