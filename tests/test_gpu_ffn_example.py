"""The example's fine-tuning step with the feed-forward block and the head without logits: every weight's gradient against
automatic differentiation of the model in 64 bits, eagerly and in a graph, and the commands."""
import os
import subprocess
import sys

import pytest
import torch

import finetune_ref as R
from test_gpu_finetune_example import ROOT, _example

pytestmark = pytest.mark.gpu


def _model(step, batch):
    """Loss and gradients in 64 bits on the CPU."""
    hq, hkv, d = step.dims
    seqs = []
    for s in range(len(batch["prompt_len"])):
        sl = slice(batch["attr_ptr"][s], batch["attr_ptr"][s + 1])
        seqs.append((int(batch["prompt_len"][s]), batch["attr_len"][sl].tolist(), batch["value_len"][sl].tolist()))
    b = R.Batch(seqs, batch["k_max"])
    w = {n: x.double().cpu().requires_grad_() for n, x in step.master.items()}
    x = w["embed"][torch.from_numpy(batch["tokens"])]
    qkv = (x @ w["qkv"]).view(b.n, hq + 2 * hkv, d)
    half = d // 2
    ang = torch.from_numpy(b.pos).double()[:, None] * (10000.0 ** (-torch.arange(half, dtype=torch.float64) / half))
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]

    def rotated(t):
        lo, hi = t[..., :half], t[..., half:]
        return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)
    q, k, v = rotated(qkv[:, :hq]), rotated(qkv[:, hq:hq + hkv]), qkv[:, hq + hkv:]
    outs = []
    for i, n in enumerate(b.len):
        sl = slice(b.off[i], b.off[i] + n)
        kk, vv = (t[sl].repeat_interleave(hq // hkv, 1).transpose(0, 1) for t in (k, v))
        score = q[sl].transpose(0, 1) @ kk.transpose(1, 2) / d ** 0.5
        score = score.masked_fill(~torch.from_numpy(b.masks[i]), -float("inf"))
        outs.append((torch.softmax(score, -1) @ vv).transpose(0, 1))
    y = x + torch.cat(outs).reshape(b.n, hq * d) @ w["out"]
    if step.inner:
        y = y + (torch.nn.functional.silu(y @ w["gate"].T) * (y @ w["up"].T)) @ w["down"].T
    head = w["head"].T if step.fused_head else w["head"]
    logits = y[torch.from_numpy(batch["rows"])] @ head
    loss = torch.nn.functional.cross_entropy(logits, torch.from_numpy(batch["targets"]))
    loss.backward()
    return loss.item(), {n: t.grad for n, t in w.items()}


@pytest.mark.parametrize("dtype, tol", [("f32", 2e-5), ("bf16", 3e-2)])
@pytest.mark.parametrize("inner, head", [(768, True), (200, False), (0, True)])
def test_gradients_of_every_weight(inner, head, dtype, tol):
    """Norm of the difference over the norm.  fp32: chains of sums of up to 768 terms; bf16: a handful of roundings of half a
    step (2^-8) in a row, weights among them."""
    ex = _example()
    batch = ex.synthetic_batch(3, n_seq=3)
    step = ex.Step(batch, dtype=dtype, inner=inner, fused_head=head)
    loss, grad = _model(step, batch)

    def check():
        torch.cuda.synchronize()
        assert abs(step.loss() - loss) <= tol * abs(loss)
        assert set(step.grad) == set(grad)
        for name, g in grad.items():
            got = step.grad[name].double().cpu()
            assert (got - g).norm() <= tol * g.norm(), name

    def run():
        step.forward()
        step.backward()
    run()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for g in step.grad.values():
            g.fill_(float("nan"))
        step.logprob.fill_(float("nan"))
        graph.replay()
        check()
        torch.ones(1000, device="cuda").sum().item()  # (the program's own work between the replays)


@pytest.mark.parametrize("args", [["--inner", "256", "--head"], ["--inner", "64", "--graph", "--dtype", "f32"], ["--head", "--graph"]])
def test_commands_run(args):
    run = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "finetune_step.py"), "--steps", "3", *args],
                         capture_output=True, text=True, timeout=100)
    assert run.returncode == 0, run.stderr[-2000:]
    assert run.stdout.count("loss") == 3 and "nan" not in run.stdout
