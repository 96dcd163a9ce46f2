"""Work lists of causal attention, on the host: tests/causal_list_driver.cpp under the address and undefined-behaviour
sanitizers. And the accumulators of the wide causal dK/dV kernel, as test_build_guard.py checks the others'."""
import os
import shutil
import subprocess

import pytest

from paper_2607_01701_amd import build as B
from test_build_guard import accumulator_faults

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_lists_cover_the_work_and_changes_are_reported(tmp_path):
    exe = str(tmp_path / "lists")
    src = [os.path.join(HERE, "causal_list_driver.cpp")] + [os.path.join(B.CSRC, s) for s in ("t2v_causal.cpp", "t2v_host.cpp")]
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-I", os.path.join(B.ROOT, "include"), *src, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok: 1200 lists"), r.stdout[-500:] + r.stderr[-2000:]


@pytest.mark.skipif(not os.path.exists(B.HIPCC) and shutil.which("hipcc") is None, reason="hipcc not available")
@pytest.mark.parametrize("flags", [[], B.CHECKED_FLAGS], ids=["product", "checked"])
def test_accumulators_are_not_moved_before_they_settle(flags, tmp_path):
    src, out = "t2v_causal_dkdv_wide.hip", tmp_path / "kernel.asm"
    r = subprocess.run([B.HIPCC, *B.HIP_FLAGS, *flags, *B.SCHED.get(src, []), "-S", "--cuda-device-only",
                        os.path.join(B.CSRC, src), "-o", str(out)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                       text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:]
    faults, n_mfma = accumulator_faults(out.read_text())
    assert n_mfma >= 64 and not faults, faults[:5]
