"""Checks on the compiler's output for the softmax attention's kernels, whose loads to LDS are asm statements: each brings the wait states
that test_ffn_asm_checks tells of, whether it loads four words a lane or one."""
import os
import subprocess

from tests.test_ffn_asm_checks import entry, scan_loads


def test_loads_to_lds_bring_their_wait_states(tmp_path):
    flags = [f for f in entry.HIPCC_FLAGS if f not in ("-shared", "-Wall")] + ["-fno-honor-nans", "-S", "--cuda-device-only"]
    runs = []
    for unit in ("softmax_bf16.hip", "softmax_bwd_bf16.hip", "softmax_f32.hip", "softmax_bwd_f32.hip"):
        out = str(tmp_path / (unit + ".s"))
        runs.append((out, subprocess.Popen(["hipcc"] + flags + [os.path.join(entry.CSRC, unit), "-o", out], stdout=subprocess.PIPE,
                                           stderr=subprocess.STDOUT, text=True)))
    for out, p in runs:
        said, _ = p.communicate()
        assert p.returncode == 0, said
        text = open(out).read()
        words = text.count("buffer_load_dword ")
        assert (words > 10) == ("bwd" in out)      # the queries' statistics
        issued, short = scan_loads(text.replace("buffer_load_dword ", "buffer_load_dwordx4 "))
        assert issued > 100 and not short, (out, issued, short[:5])
