"""The example's fine-tuning step: every weight's gradient against automatic differentiation of the model in 64 bits on the
CPU, and a training run eagerly and in a graph."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import finetune_ref as R

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("finetune_step", os.path.join(ROOT, "examples", "finetune_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _model(step, batch):
    """Loss and gradients in 64 bits on the CPU; the mask and positions are the oracle's."""
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
        score = q[sl].transpose(0, 1) @ kk.transpose(1, 2) / np.sqrt(d)
        score = score.masked_fill(~torch.from_numpy(b.masks[i]), -float("inf"))
        outs.append((torch.softmax(score, -1) @ vv).transpose(0, 1))
    y = x + torch.cat(outs).reshape(b.n, hq * d) @ w["out"]
    logits = y[torch.from_numpy(batch["rows"])] @ w["head"]
    loss = torch.nn.functional.cross_entropy(logits, torch.from_numpy(batch["targets"]))
    loss.backward()
    return loss.item(), {n: t.grad for n, t in w.items()}


@pytest.mark.parametrize("dtype, tol", [("f32", 2e-5), ("bf16", 3e-2)])
def test_gradients_of_every_weight(dtype, tol):
    """Norm of the difference over the norm.  fp32: chains of sums of up to 512 terms; bf16: a handful of roundings of half a
    step (2^-8) in a row, weights among them."""
    ex = _example()
    batch = ex.synthetic_batch(3, n_seq=3)
    step = ex.Step(batch, dtype=dtype)
    step.forward()
    step.backward()
    loss, grad = _model(step, batch)
    assert abs(step.loss() - loss) <= tol * abs(loss)
    for name, g in grad.items():
        got = step.grad[name].double().cpu()
        assert (got - g).norm() <= tol * g.norm(), name


def test_training_eagerly_and_in_a_graph():
    ex = _example()
    batch = ex.synthetic_batch(0)
    eager, captured = ex.Step(batch), ex.Step(batch)
    eager.run()
    first = eager.loss()
    captured.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    for _ in range(14):
        eager.run()
        graph.replay()
        torch.cuda.synchronize()
        assert abs(eager.loss() - captured.loss()) <= 1e-2 * abs(first)  # (index_add_ adds in any order)
    assert eager.loss() < 0.8 * first and eager.accuracy() > 0
