"""Checks on the compiler's output for the gated feed-forward block's product kernels, whose loads to LDS are asm statements.

The compiler does not know what such a statement holds, so it puts no wait states before it.  A buffer load needs one behind the
write of m0 that it reads, and five behind a vector instruction that wrote its descriptor's scalar registers, wherever the
compiler has placed that instruction: the statement itself has to bring them."""
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
import __graft_entry__ as entry      # noqa: E402


def scan_loads(text):
    """(number of hand-written loads to LDS, those with fewer wait states in their statement than they need)."""
    issued, short, inside, states, m0 = 0, [], False, 0, None
    for ln, line in enumerate(text.split("\n"), 1):
        t = line.strip()
        if t.startswith(";;#ASMSTART"):
            inside, states, m0 = True, 0, None
        elif t.startswith(";;#ASMEND"):
            inside = False
        elif inside and t and t[0] not in ";.":
            op = t.split()[0]
            if op == "buffer_load_dwordx4" and t.endswith(" lds"):
                issued += 1
                if states < 5 or m0 is None or states - m0 < 1:
                    short.append("line %d: %s" % (ln, t))
            states += int(t.split()[1], 0) + 1 if op == "s_nop" else 1
            if op == "s_mov_b32" and t.split()[1] == "m0,":
                m0 = states
    return issued, short


def test_scanner_counts_wait_states():
    def statement(nop):
        return "\t;;#ASMSTART\n\ts_mov_b32 m0, s4\n\ts_nop %d\n\tbuffer_load_dwordx4 v1, s[0:3], 0 offen lds\n\t;;#ASMEND\n" % nop
    assert scan_loads(statement(3)) == (1, [])
    assert scan_loads(statement(2))[0] == 1 and "line 4" in scan_loads(statement(2))[1][0]


@pytest.mark.parametrize("unit", ["ffn_bf16.hip", "ffn_f16.hip", "ffn_f32.hip"])
def test_loads_to_lds_bring_their_wait_states(unit, tmp_path):
    flags = [f for f in entry.HIPCC_FLAGS if f not in ("-shared", "-Wall")] + ["-S", "--cuda-device-only"]
    out = str(tmp_path / (unit + ".s"))
    r = subprocess.run(["hipcc"] + flags + [os.path.join(entry.CSRC, unit), "-o", out], stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    issued, short = scan_loads(open(out).read())
    assert issued > 100, issued
    assert not short, short[:5]
