"""Shapes, cuts and workspaces of the feed-forward block's and the vocabulary head's products, on the host."""
import os
import shutil
import subprocess

import pytest

from paper_2604_26209_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(not shutil.which("g++"), reason="g++ not installed")
def test_plans(tmp_path):
    exe = str(tmp_path / "product_plans")
    cmd = ["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2604_26209_amd", "csrc"),
           os.path.join(ROOT, "tests", "native", "product_plans_main.cpp"), "-o", exe]
    build = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert build.returncode == 0, build.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "no finding" in run.stdout, run.stderr[-2000:]


@pytest.mark.parametrize("dtype", [B.HPD_BF16, B.HPD_F32])
@pytest.mark.parametrize("width, other", [(64, 40), (256, 520), (2048, 5504), (4096, 12288), (4096, 2057), (1152, 50021)])
def test_a_workspace_is_enough_for_fewer_rows(width, other, dtype):
    """What a call of n rows needs is at most what is reported for them, so reports that never fall with n hold every smaller call."""
    cfg = B.hpd_ffn_config(width, other // 8 * 8, dtype, B.HPD_ACT_SILU)
    last = (0,) * 4
    for n in [*range(1, 1100), *range(2000, 2100), 4095, 4096, 4097, 8192, 20000, 1 << 18]:
        now = B.hpd_gated_ffn_workspace(cfg, n) + B.hpd_head_logprobs_workspace(dtype, n, width, other)
        assert all(a >= b for a, b in zip(now, last)), n
        last = now


def test_workspaces_of_short_contractions():
    """A part has four stages of 64 elements (fp32: 32) at least: fewer than eight stages leave nothing but what the products have for each
    other, eight (504 and 2 x 248 elements of bf16, 248 of fp32) two parts of the result."""
    rows, width = 5000, 4096
    for inner, parts in ((448, 0), (504, 2)):
        cfg = B.hpd_ffn_config(width, inner, B.HPD_BF16, B.HPD_ACT_SILU)
        assert B.hpd_gated_ffn_workspace(cfg, rows)[0] == rows * inner * 2 + parts * rows * width * 4
    for inner, parts in ((224, 0), (248, 2)):
        cfg = B.hpd_ffn_config(width, inner, B.HPD_BF16, B.HPD_ACT_SILU)
        assert B.hpd_gated_ffn_workspace(cfg, rows)[1] == 3 * rows * inner * 2 + parts * rows * width * 4
    # rows' sums of 100 tiles and the target's logit, or two parts of the logits up to 128 MB
    assert B.hpd_head_logprobs_workspace(B.HPD_F32, rows, 224, 6400)[0] == rows * (100 * 16 + 4)
    assert B.hpd_head_logprobs_workspace(B.HPD_F32, rows, 248, 6400)[0] == 128 << 20
