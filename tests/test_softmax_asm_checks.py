"""Checks on the compiler's output for the softmax attention's kernels, whose loads to LDS are asm statements: each brings the wait states
that test_ffn_asm_checks tells of, whether it loads four words a lane or one."""
import subprocess

import pytest

from tests.test_ffn_asm_checks import entry, scan_loads

# a kernel of every kind: the units of all widths hold the same statements and take minutes
FORWARD = '''
#include "kernels.h"
#include "softmax_kernels.inc"
namespace aa {
hipError_t some(const SoftmaxArgs& a, SoftmaxPass pass, hipStream_t st) {
  hipError_t err = launch_forward<ElemBF16, 64>(a, pass, 1, st);
  return err == hipSuccess ? launch_forward<ElemF32, 128>(a, pass, 1, st) : err;
}
}
'''
BACKWARD = '''
#include "kernels.h"
#include "softmax_bwd_kernels.inc"
namespace aa {
hipError_t some(const SoftmaxArgs& a, SoftmaxPass pass, hipStream_t st) {
  hipError_t err = launch_backward<ElemF16, 128>(a, pass, 1, st);
  return err == hipSuccess ? launch_backward<ElemF32x3, 48>(a, pass, 1, st) : err;
}
}
'''


@pytest.mark.parametrize("source", [FORWARD, BACKWARD], ids=["forward", "backward"])
def test_loads_to_lds_bring_their_wait_states(source, tmp_path):
    flags = [f for f in entry.HIPCC_FLAGS if f not in ("-shared", "-Wall")] + ["-fno-honor-nans", "-S", "--cuda-device-only", "-I", entry.CSRC]
    unit, out = tmp_path / "some.hip", tmp_path / "some.s"
    unit.write_text(source)
    r = subprocess.run(["hipcc"] + flags + [str(unit), "-o", str(out)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    text = out.read_text()
    assert (text.count("buffer_load_dword ") > 10) == (source is BACKWARD)      # the queries' statistics
    issued, short = scan_loads(text.replace("buffer_load_dword ", "buffer_load_dwordx4 "))
    assert issued > 100 and not short, (issued, short[:5])
