"""Fine-tuning steps of a one-layer attention model under the HPD mask, through the library's operators: rotation, masked
attention, log probabilities of the value tokens, and their gradients; the projections are plain matrix products.

    python examples/finetune_step.py [--steps 20] [--dtype bf16] [--graph] [--inner 768] [--head]

--inner puts a gated feed-forward block of that inner width behind the attention; --head takes the log probabilities from the
hidden states and the vocabulary's weights, without logits in memory.
The task is synthetic: the first token of an attribute's name decides its value's tokens.  Every step updates the weights by
plain gradient descent; with --graph the whole step is captured in a HIP graph once and replayed.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_26209_amd import binding as B  # noqa: E402


def synthetic_batch(seed, n_seq=8, prompt=48, n_attr=6, k_max=8, vocab=512):
    """Lengths, tokens and, per row that predicts a value token, the row and the token."""
    rng = np.random.default_rng(seed)
    prompt_len = rng.integers(prompt // 2, prompt + 1, n_seq)
    attr_ptr = np.arange(n_seq + 1) * n_attr
    attr_len = rng.integers(1, 4, n_seq * n_attr)
    value_len = rng.integers(1, k_max + 1, n_seq * n_attr)
    tokens, rows, targets = [], [], []
    for s in range(n_seq):
        tokens += rng.integers(0, vocab, prompt_len[s]).tolist()
        for n in range(attr_ptr[s], attr_ptr[s + 1]):
            name = rng.integers(0, vocab, attr_len[n])
            tokens += name.tolist()
            for k in range(value_len[n]):  # value token k follows from the name
                rows.append(len(tokens) - 1)
                targets.append(int((name[-1] * 7 + 13 * k) % vocab))
                tokens.append(targets[-1])
    return dict(prompt_len=prompt_len, attr_ptr=attr_ptr, attr_len=attr_len, value_len=value_len, k_max=k_max,
                tokens=np.array(tokens), rows=np.array(rows), targets=np.array(targets))


class Step:
    """Weights, activations and gradients of the model for one batch; run() is one training step."""

    def __init__(self, batch, vocab=512, width=256, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype="bf16", rate=0.5, top=3,
                 seed=0, inner=0, fused_head=False):
        dev, td = "cuda", torch.float32 if dtype == "f32" else torch.bfloat16
        self.dt = B.HPD_F32 if dtype == "f32" else B.HPD_BF16
        hq, hkv, d = n_q_heads, n_kv_heads, head_dim
        self.rate, self.top, self.vocab, self.dims = rate, top, vocab, (hq, hkv, d)
        self.width, self.inner, self.fused_head = width, inner, fused_head
        cfg = B.hpd_finetune_config(hq, hkv, d, self.dt, 10000.0, batch["k_max"], 0)
        self.layout = B.hpd_build_finetune_layout(cfg, batch["prompt_len"], batch["attr_ptr"], batch["attr_len"],
                                                  batch["value_len"])
        self.tokens = torch.from_numpy(batch["tokens"]).to(dev)
        self.rows = torch.from_numpy(batch["rows"]).to(dev)
        self.targets = torch.from_numpy(batch["targets"]).to(dev, torch.int32)
        n, m = len(batch["tokens"]), len(batch["rows"])
        assert n == self.layout.counts()[B.HPD_FTC_N_TOKENS]
        gen = torch.Generator().manual_seed(seed)
        self.master = {name: (torch.randn(shape, generator=gen) * std).to(dev) for name, shape, std in (
            ("embed", (vocab, width), 0.5), ("qkv", (width, (hq + 2 * hkv) * d), width ** -0.5),
            ("out", (hq * d, width), (hq * d) ** -0.5),
            ("head", (vocab, width) if fused_head else (width, vocab), width ** -0.5))}
        if inner:
            self.master |= {name: (torch.randn(shape, generator=gen) * shape[1] ** -0.5).to(dev) for name, shape in (
                ("gate", (inner, width)), ("up", (inner, width)), ("down", (width, inner)))}

        def empty(*shape, t=td):
            return torch.empty(shape, dtype=t, device=dev)

        self.q, self.k, self.o, self.d_o = empty(n, hq, d), empty(n, hkv, d), empty(n, hq, d), empty(n, hq, d)
        self.dq, self.dk, self.d_qkv = empty(n, hq, d), empty(n, hkv, d), empty(n, hq + 2 * hkv, d)
        self.attn_lse = empty(hq, n, t=torch.float32)
        self.logprob, self.lse, self.entropy = (empty(m, t=torch.float32) for _ in range(3))
        self.top_id, self.top_logprob = empty(m, top, t=torch.int32), empty(m, top, t=torch.float32)
        self.g_logprob = torch.full((m,), -1.0 / m, device=dev)
        self.ws = [B.alloc_finetune_workspace(self.layout, b) for b in (False, True)]
        self.loss_ws = empty(max(1, B.hpd_token_logprobs_workspace(self.dt, m, vocab, top)), t=torch.uint8)
        self.td = td
        if inner:
            self.ffn = B.hpd_ffn_config(width, inner, self.dt, B.HPD_ACT_SILU)
            self.ffn_out, self.d_ffn_in = empty(n, width), empty(n, width)
            self.gate, self.up = empty(n, inner), empty(n, inner)
            self.d_ffn = empty(inner, width), empty(inner, width), empty(width, inner)
            self.ffn_ws = [B.alloc_ffn_workspace(self.ffn, n, b) for b in (False, True)]
        if fused_head:
            self.d_rows, self.d_head = empty(m, width), empty(vocab, width)
            self.head_ws = [B.alloc_head_workspace(self.dt, m, width, vocab, b) for b in (False, True)]

    def heads(self, x):
        hq, hkv, _ = self.dims
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]

    def forward(self):
        hq, hkv, d = self.dims
        self.w = {name: w.to(self.td) for name, w in self.master.items()}
        self.x = self.w["embed"][self.tokens]
        qkv = (self.x @ self.w["qkv"]).view(-1, hq + 2 * hkv, d)
        q, k, self.v = self.heads(qkv)
        row = qkv.stride(0)
        B.hpd_finetune_rotate(self.layout, 0, q, k, self.q, self.k, B.hpd_finetune_strides(q=row, k=row))
        B.hpd_finetune_attention(self.layout, self.q, self.k, self.v, self.o, self.attn_lse, self.ws[0],
                                 B.hpd_finetune_strides(v=row))
        self.y = self.x + self.o.view(-1, hq * d) @ self.w["out"]
        z = self.y
        if self.inner:
            B.hpd_gated_ffn(self.ffn, len(z), z, self.w["gate"], self.w["up"], self.w["down"], self.ffn_out, self.gate,
                            self.up, self.ffn_ws[0])
            z = z + self.ffn_out
        self.hidden = z[self.rows]
        if self.fused_head:
            B.hpd_head_logprobs(self.dt, len(self.hidden), self.width, self.vocab, self.hidden, self.width, self.w["head"],
                                self.width, self.targets, self.logprob, self.lse, self.entropy, self.head_ws[0])
            return
        self.logits = self.hidden @ self.w["head"]
        m = self.logits.shape[0]
        B.hpd_token_logprobs(self.dt, m, self.vocab, self.vocab, self.logits, self.targets, self.top, self.logprob, self.lse,
                             self.entropy, self.top_id, self.top_logprob, self.loss_ws)

    def backward(self):
        hq, hkv, d = self.dims
        self.grad = {}
        if self.fused_head:
            d_rows, self.grad["head"] = self.d_rows, self.d_head
            B.hpd_head_logprobs_backward(self.dt, len(self.hidden), self.width, self.vocab, self.hidden, self.width,
                                         self.w["head"], self.width, self.targets, self.lse, None, self.g_logprob, None, d_rows,
                                         self.width, self.d_head, self.width, self.head_ws[1])
        else:
            m = self.logits.shape[0]
            B.hpd_token_logprobs_backward(self.dt, m, self.vocab, self.vocab, self.logits, self.targets, self.lse, None,
                                          self.g_logprob, None, self.logits, self.vocab)  # in place
            d_rows = self.logits @ self.w["head"].t()
            self.grad["head"] = self.hidden.t() @ self.logits
        dy = torch.zeros_like(self.y).index_copy_(0, self.rows, d_rows)
        if self.inner:
            B.hpd_gated_ffn_backward(self.ffn, len(dy), self.y, self.w["gate"], self.w["up"], self.w["down"], self.gate, self.up,
                                     dy, self.d_ffn_in, *self.d_ffn, self.ffn_ws[1])
            dy = dy + self.d_ffn_in
            self.grad |= dict(zip(("gate", "up", "down"), self.d_ffn))
        torch.matmul(dy, self.w["out"].t(), out=self.d_o.view(-1, hq * d))
        dq, dk, dv = self.heads(self.d_qkv)
        row = self.d_qkv.stride(0)
        B.hpd_finetune_attention_backward(self.layout, self.q, self.k, self.v, self.o, self.attn_lse, self.d_o, self.dq,
                                          self.dk, dv, self.ws[1], B.hpd_finetune_strides(v=row, v_out=row))
        B.hpd_finetune_rotate(self.layout, 1, self.dq, self.dk, dq, dk, B.hpd_finetune_strides(q_out=row, k_out=row))
        d_qkv = self.d_qkv.view(-1, row)
        dx = dy + d_qkv @ self.w["qkv"].t()
        self.grad |= dict(embed=torch.zeros_like(self.master["embed"]).index_add_(0, self.tokens, dx.float()),
                          qkv=self.x.t() @ d_qkv, out=self.o.view(-1, hq * d).t() @ dy)

    def update(self):
        for name, w in self.master.items():
            w.sub_(self.grad[name].float(), alpha=self.rate)

    def run(self):
        self.forward()
        self.backward()
        self.update()

    def loss(self):
        return -self.logprob.mean().item()

    def accuracy(self):
        return (self.top_id[:, 0] == self.targets).float().mean().item()


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    p.add_argument("--graph", action="store_true")
    p.add_argument("--inner", type=int, default=0)
    p.add_argument("--head", action="store_true")
    args = p.parse_args()
    step = Step(synthetic_batch(0), dtype=args.dtype, inner=args.inner, fused_head=args.head)
    run = step.run
    if args.graph:
        step.run()  # (libraries set themselves up)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step.run()
        run = graph.replay
    for i in range(args.steps):
        run()
        right = "" if args.head else f", most likely token right {100 * step.accuracy():.1f} %"
        print(f"step {i}: loss {step.loss():.4f}, entropy {step.entropy.mean().item():.3f}{right}", flush=True)


if __name__ == "__main__":
    main()
