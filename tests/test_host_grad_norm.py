"""acc_get_grad_norm() after iterations that measured a norm, were refused or failed: the real executor, built for the host with g++ under AddressSanitizer and UBSan
against the stand-in runtime (tests/hoststub)."""
import os
import subprocess

import synth as S
from test_host_executor import CSRC, STUB, spec_file


def test_the_norm_is_that_of_the_last_iteration_or_none(tmp_path):
    exe = str(tmp_path / "clip_check")
    srcs = [os.path.join(CSRC, f) for f in ("graph.cpp", "plan.cpp", "engine.hip")] + [os.path.join(STUB, f) for f in ("stub_runtime.cpp", "clip_check.cpp")]
    subprocess.check_call(["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined", "-fno-omit-frame-pointer", "-fno-sanitize-recover=undefined",
                           "-I", STUB, "-x", "c++"] + srcs + ["-o", exe])
    p = subprocess.run([exe, spec_file(tmp_path, S.bottleneck_unit())], capture_output=True, text=True, timeout=120)
    assert p.returncode == 0 and not p.stderr, p.stderr
    assert p.stdout.splitlines() == ["before any iteration: -6",
                                     "measured: 0 0",
                                     "refused: -1 0",            # nothing ran: the last iteration is the one before
                                     "failed: 1 -6",
                                     "again: 0 0"]
