"""Checks without a GPU that no block of the keys' kernel of softmax attention passes a barrier, or ends, while loads to LDS may be under way that
it has not waited for: on the compiler's output, over every path through a kernel.  The loads are asm statements, so the compiler puts no wait
for them anywhere; a wait that stands in a loop alone is none for a block whose range of queries is empty and goes past the loop."""
import re
import subprocess

import pytest

from tests.softmax_plans import CAUSAL, empty_ranges, plans      # noqa: F401
from tests.test_ffn_asm_checks import entry

# all that hold values in LDS (65 to 128 channels of 16 bits) and two that do not; blocks of two waves, of four, and of four with two on the same rows
KERNELS = ("ElemBF16, 80, 4, 1, 2", "ElemF16, 96, 4, 2, 2", "ElemBF16, 128, 4, 1, 2", "ElemF16, 80, 2, 1, 1", "ElemBF16, 96, 4, 1, 1",
           "ElemF16, 128, 4, 1, 1", "ElemBF16, 64, 4, 1, 2", "ElemF32x3, 48, 2, 1, 1")
SOURCE = '''
#include "kernels.h"
#include "softmax_bwd_kernels.inc"
namespace aa {
hipError_t some(const SoftmaxArgs& a, hipStream_t st) {
  hipError_t err = hipSuccess;
%s
  return err;
}
}
'''


def functions(text):
    """(name, its lines) of every kernel in the compiler's output."""
    for m in re.finditer(r"^(\S+):\s*; @\1\n(.*?)^\.Lfunc_end", text, re.S | re.M):
        yield m.group(1), [line.split(";")[0].strip() for line in m.group(2).split("\n") if not line.strip().startswith(";;")]


def passed_over(lines):
    """Lines with a barrier or an end of the program that some path reaches with a load to LDS behind it and no wait for all loads since."""
    labels = {line[:-1]: n for n, line in enumerate(lines) if re.fullmatch(r"\.\w+:", line)}
    found, seen, todo = set(), set(), [(0, False)]
    while todo:
        n, pending = todo.pop()
        while n < len(lines) and (n, pending) not in seen:
            seen.add((n, pending))
            op, _, rest = lines[n].partition(" ")
            op, rest = op.strip(), rest.strip()
            if op.startswith("buffer_load") and rest.endswith(" lds"):
                pending = True
            elif op == "s_waitcnt" and "vmcnt(0)" in rest:
                pending = False
            elif op in ("s_barrier", "s_endpgm") and pending:
                found.add("%d: %s" % (n, lines[n]))
            if op == "s_endpgm":
                break
            if op == "s_branch":
                n = labels[rest]
                continue
            assert op not in ("s_setpc_b64", "s_swappc_b64", "s_call_b64"), op
            if op.startswith("s_cbranch"):
                todo.append((labels[rest], pending))
            n += 1
    return sorted(found)


def test_the_scan_follows_branches():
    loop = ["buffer_load_dwordx4 v1, s[0:3], 0 offen lds", "s_cbranch_scc1 .LBB0_2", ".LBB0_1:", "s_waitcnt vmcnt(0) lgkmcnt(0)", "s_barrier",
            "s_cbranch_scc0 .LBB0_1", ".LBB0_2:", "%s", "s_barrier", "s_endpgm"]
    assert passed_over([x % "s_nop 0" if "%" in x else x for x in loop]) == ["8: s_barrier", "9: s_endpgm"]
    assert passed_over([x % "s_waitcnt vmcnt(0)" if "%" in x else x for x in loop]) == []
    assert passed_over([x % "s_waitcnt vmcnt(3)" if "%" in x else x for x in loop]) == ["8: s_barrier", "9: s_endpgm"]


def test_no_barrier_is_passed_with_loads_under_way(tmp_path):
    flags = [f for f in entry.HIPCC_FLAGS if f not in ("-shared", "-Wall")] + ["-fno-honor-nans", "-S", "--cuda-device-only", "-I", entry.CSRC]
    # a unit for each, compiled side by side
    runs = []
    for i, k in enumerate(KERNELS):
        unit, out = tmp_path / ("some%d.hip" % i), tmp_path / ("some%d.s" % i)
        unit.write_text(SOURCE % ("  err = launch_keys<%s>(a, 1, st);" % k))
        runs.append((k, out, subprocess.Popen(["hipcc"] + flags + [str(unit), "-o", str(out)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                              text=True)))
    for k, out, run in runs:
        said, _ = run.communicate()
        assert run.returncode == 0, said
        kernels = [lines for name, lines in functions(out.read_text()) if "softmax_dkv" in name]
        assert len(kernels) == 1 and sum(line.endswith(" lds") for line in kernels[0]) >= 4, k
        assert passed_over(kernels[0]) == [], k


@pytest.mark.parametrize("case", CAUSAL, ids=lambda c: "x".join(map(str, c)))
def test_causal_calls_have_empty_ranges_of_queries(plans, case):      # noqa: F811
    """The sizes that the GPU tests of such ranges go by."""
    assert empty_ranges(plans(*case), *case) > 0


@pytest.mark.parametrize("case", [(3, 4, 2, 150, 200, 80, 0), (3, 4, 2, 150, 200, 128, 0), (8, 8, 8, 600, 600, 96, 0)], ids=lambda c: "x".join(map(str, c)))
def test_calls_with_sequences_of_no_queries_share_their_keys(plans, case):      # noqa: F811
    assert plans(*case)["together"]
