"""What the calls of the fine-tuning operators refuse before a kernel is launched (CPU build of their host side with the
launchers replaced, tests/native/finetune_calls_main.cpp), and batches that no launch can hold."""
import os
import subprocess

import numpy as np
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


@pytest.mark.parametrize("dtype, heads, most", [("f32", (32, 8), 2 ** 17 - 1), ("bf16", (32, 8), 2 ** 19 - 1),
                                                ("f32", (16, 16), 2 ** 18 - 1), ("bf16", (16, 16), 2 ** 20 - 1)])
def test_batches_of_more_sequences_than_a_launch_holds(dtype, heads, most):
    """A launch has less than 2^32 threads: 256 for every sequence and query head at least, in fp32 1024.  The tokens are
    few enough."""
    from paper_2604_26209_amd import binding as B
    cfg = B.hpd_finetune_config(*heads, 64, B.HPD_F32 if dtype == "f32" else B.HPD_BF16, 10000.0, 4, B.HPD_FLAG_HOST_ONLY)

    def build(n):
        return B.hpd_build_finetune_layout(cfg, np.ones(n, np.int32), np.zeros(n + 1, np.int32), [], [])
    assert build(most).counts()[B.HPD_FTC_N_SEQ] == most
    with pytest.raises(B.HpdError) as e:
        build(most + 1)
    assert e.value.status == B.HPD_E_OVERFLOW


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_heads_of_a_token_beyond_32_bits(dtype):
    """A head's place in its token is a 32-bit number of bytes or elements in the kernels."""
    from paper_2604_26209_amd import binding as B

    def build(heads):
        cfg = B.hpd_finetune_config(heads, 1, 128, B.HPD_F32 if dtype == "f32" else B.HPD_BF16, 10000.0, 4, B.HPD_FLAG_HOST_ONLY)
        return B.hpd_build_finetune_layout(cfg, [1], [0, 0], [], [])
    assert build(2 ** 20).counts()[B.HPD_FTC_N_TOKENS] == 1
    with pytest.raises(B.HpdError) as e:
        build(2 ** 23 + 2 ** 10)
    assert e.value.status == B.HPD_E_OVERFLOW
