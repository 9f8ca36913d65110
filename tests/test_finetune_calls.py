"""What the calls of the fine-tuning operators refuse before a kernel is launched (CPU build of their host side with the
launchers replaced, tests/native/finetune_calls_main.cpp)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_calls_are_run_or_refused_as_declared(tmp_path):
    exe = str(tmp_path / "finetune_calls")
    cmd = [HIPCC, "-O1", "-g", "-std=c++20", "-x", "hip", "--offload-arch=gfx950", "--offload-host-only",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2604_26209_amd", "csrc"),
           os.path.join(ROOT, "paper_2604_26209_amd", "csrc", "hpd_finetune_host.cpp"),
           os.path.join(ROOT, "tests", "native", "finetune_calls_main.cpp"), "-o", exe]
    build = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert build.returncode == 0, build.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "as declared" in run.stdout, (run.stdout + run.stderr)[-2000:]
