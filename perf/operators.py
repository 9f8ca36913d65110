"""The operators of a fine-tuning step under the HPD mask, as cases to be measured.

Five operators: the rotation of queries and keys at the position IDs of packed training sequences
(and its inverse, for gradients), attention over them under the fine-tuning mask (paper Section
4.4), its gradient, the log probabilities of given tokens with entropy and top alternatives, and
the gradient of those.  ``run`` computes them in elementary torch operations where ``own`` is
false and through the library where it is true.

Sizes: heads, header / document / value lengths and attribute counts are those of the benchmark
configurations (``workloads.config``) and of the tests' ragged batches; vocabularies are generic.
"""
import math
import random

import numpy as np
import torch

own = False

# the largest cases that are drawn: forward operations of an attention (a gradient has 2.5 times as many), bytes of logits
F32_FLOPS, BF16_FLOPS = 4e11, 2.1e12
LOGIT_BYTES = 1.58e9
SEQUENCE_OPS = ("rotate", "attn", "attn_grad")


def listed():
    return [
        # queries and keys of a training batch, views of one projection's output
        dict(name="rotate_batch", op="rotate", inverse=False, dtype="bf16", hq=32, hkv=8, d=128, base=500000.0,
             k_max=16, n_seq=32, prompt_lo=300, prompt_hi=576, n_attr=16, fused=True, lens=2),
        # gradients of the small fp32 layer, turned back
        dict(name="rotate_back_f32", op="rotate", inverse=True, dtype="f32", hq=4, hkv=4, d=64, base=10000.0,
             k_max=8, n_seq=16, prompt_lo=16, prompt_hi=700, n_attr=8, fused=False, lens=4),
        # one short sequence, the smallest call: a header, four attributes
        dict(name="attn_one_short", op="attn", dtype="bf16", hq=32, hkv=8, d=128, base=500000.0, k_max=8,
             n_seq=1, prompt_lo=40, prompt_hi=40, n_attr=4, fused=False, lens=1),
        # two long stacked documents, 96 attributes, 64 query heads
        dict(name="attn_long", op="attn", dtype="bf16", hq=64, hkv=8, d=128, base=500000.0, k_max=32,
             n_seq=4, prompt_lo=4000, prompt_hi=4224, n_attr=96, fused=False, lens=3),
        # the small fp32 layer, ragged
        dict(name="attn_f32", op="attn", dtype="f32", hq=4, hkv=4, d=64, base=10000.0, k_max=8,
             n_seq=16, prompt_lo=16, prompt_hi=700, n_attr=8, fused=False, lens=4),
        # gradients of a training batch of single documents with 16 attributes each; v and dv in the
        # projection's output and its gradient
        dict(name="attn_grad_batch", op="attn_grad", dtype="bf16", hq=32, hkv=8, d=128, base=500000.0, k_max=16,
             n_seq=32, prompt_lo=300, prompt_hi=576, n_attr=16, fused=True, lens=2),
        # ... of the long sequences
        dict(name="attn_grad_long", op="attn_grad", dtype="bf16", hq=64, hkv=8, d=128, base=500000.0, k_max=32,
             n_seq=2, prompt_lo=4000, prompt_hi=4224, n_attr=96, fused=False, lens=5),
        # ... of the small fp32 layer
        dict(name="attn_grad_f32", op="attn_grad", dtype="f32", hq=4, hkv=4, d=64, base=10000.0, k_max=8,
             n_seq=16, prompt_lo=16, prompt_hi=700, n_attr=8, fused=False, lens=4),
        # the value tokens of a training batch over a large padded vocabulary
        dict(name="logprobs_batch", op="logprobs", dtype="bf16", rows=6144, vocab=130013, stride=130048, top=1),
        # few fp32 rows, many alternatives: the teacher's side of a distillation, token by token
        dict(name="logprobs_f32_few", op="logprobs", dtype="f32", rows=3, vocab=150001, stride=150001, top=20),
        # the loss' gradient over the value tokens of a batch
        dict(name="logprobs_grad_batch", op="logprobs_grad", dtype="bf16", rows=4096, vocab=32000, stride=32000,
             entropy=False),
        # with an entropy term, fp32, an odd vocabulary
        dict(name="logprobs_grad_f32", op="logprobs_grad", dtype="f32", rows=700, vocab=50021, stride=50021,
             entropy=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotate", "attn", "attn", "attn_grad", "attn_grad", "logprobs", "logprobs_grad"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op in SEQUENCE_OPS:
        hq, hkv, d = rng.choice([(4, 4, 64), (8, 2, 64), (32, 8, 128), (64, 8, 128), (40, 8, 128), (16, 16, 128),
                                 (12, 2, 96), (6, 1, 80)])
        cap = (BF16_FLOPS if dtype == "bf16" else F32_FLOPS) / (1.0 if op == "attn" else 2.0)
        while True:
            hi = _log_int(rng, 8, 9000)
            case = dict(op=op, dtype=dtype, hq=hq, hkv=hkv, d=d, base=rng.choice([10000.0, 500000.0]),
                        k_max=rng.choice([7, 8, 12, 16, 32]), n_seq=_log_int(rng, 1, 64),
                        prompt_lo=rng.randint(0, hi), prompt_hi=hi, n_attr=_log_int(rng, 1, 96),
                        fused=rng.random() < 0.5, lens=rng.randint(10, 10 ** 6))
            if op == "rotate":
                case["inverse"] = rng.random() < 0.5
            prompt, attr_ptr, attr_len, value_len = _lengths(case)
            n = sum(prompt) + sum(attr_len) + sum(value_len)
            if 4.0 * d * hq * _pairs(case) <= cap and n * hq * d <= 2 ** 28:
                return case
    top = rng.choice([0, 1, 5, 8, 20, 50]) if op == "logprobs" else 0
    while True:
        vocab, rows = _log_int(rng, 200, 160000), _log_int(rng, 1, 8192)
        stride = vocab + rng.choice([0, 0, 1, 24])
        if rows * stride * (2 if dtype == "bf16" else 4) * (4 + max(top, 1)) <= 5 * LOGIT_BYTES:
            break
    case = dict(op=op, dtype=dtype, rows=rows, vocab=vocab, stride=stride)
    if op == "logprobs":
        case["top"] = top
    else:
        case["entropy"] = rng.random() < 0.5
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _lengths(case):
    """Prompt, attribute-name and value lengths of the case's sequences (host integers)."""
    rng = random.Random(case["lens"])
    prompt, attr_ptr, attr_len, value_len = [], [0], [], []
    for _ in range(case["n_seq"]):
        prompt.append(rng.randint(case["prompt_lo"], case["prompt_hi"]))
        for _ in range(case["n_attr"]):
            attr_len.append(rng.randint(1, 4))
            value_len.append(rng.randint(0, case["k_max"]))
        attr_ptr.append(len(attr_len))
    return prompt, attr_ptr, attr_len, value_len


def _sequences(case):
    """Per sequence: position IDs and ranks of its tokens (NumPy).  A key is seen by the queries
    that do not precede it and whose rank is no lower: rank k for the k-th token of a value, 0
    for prompt and attribute names."""
    prompt, attr_ptr, attr_len, value_len = _lengths(case)
    out = []
    for s, p in enumerate(prompt):
        pos, rank, at = list(range(p)), [0] * p, p
        for i, n in enumerate(range(attr_ptr[s], attr_ptr[s + 1])):
            shift = i * case["k_max"]
            pos += range(at + shift, at + shift + attr_len[n])
            rank += [0] * attr_len[n]
            at += attr_len[n]
            pos += range(at + shift, at + shift + value_len[n])
            rank += range(1, value_len[n] + 1)
        out.append((np.asarray(pos, dtype=np.int64), np.asarray(rank, dtype=np.int64)))
    return out


def _pairs(case):
    """(query, key) pairs that the mask leaves, all sequences."""
    total = 0
    for _, rank in _sequences(case):
        seen = np.zeros(case["k_max"] + 1, dtype=np.int64)
        first = int((rank == 0).argmin()) if rank.size and (rank != 0).any() else rank.size
        total += first * (first + 1) // 2
        seen[0] = first
        for r in rank[first:].tolist():
            seen[r] += 1
            total += int(seen[:r + 1].sum())
    return total


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _heads(buf, case):
    hq, hkv = case["hq"], case["hkv"]
    return buf[:, :hq], buf[:, hq:hq + hkv], buf[:, hq + hkv:]


def _qkv_buffers(case, n, make):
    """What belongs to q, k and v of n tokens: three tensors, or views of one."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["fused"]:
        return _heads(make((n, hq + 2 * hkv, d)), case)
    return make((n, hq, d)), make((n, hkv, d)), make((n, hkv, d))


def _make_inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = _dtype(case)

    def normal(shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dt)

    st = dict(case=case)
    if case["op"] in SEQUENCE_OPS:
        seqs = _sequences(case)
        n = sum(p.size for p, _ in seqs)
        q, k, st["v"] = _qkv_buffers(case, n, normal)
        if case["op"] != "rotate":  # the rotation has written its results next to each other
            q, k = q.contiguous(), k.contiguous()
        st["q"], st["k"] = q, k
        st["seqs"] = [(torch.from_numpy(p).cuda(), torch.from_numpy(r).cuda()) for p, r in seqs]
        if case["op"] == "attn_grad":
            st["d_out"] = normal((n, case["hq"], case["d"]))
        return st
    rows, vocab, stride = case["rows"], case["vocab"], case["stride"]
    buf = torch.empty((rows, stride), dtype=dt, device="cuda")
    for a in range(0, rows, 512):
        b = min(a + 512, rows)
        buf[a:b] = (torch.randn((b - a, stride), generator=gen, device="cuda") * 2.5).to(dt)
    x = buf[:, :vocab]
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    at = torch.arange(rows, device="cuda")
    # every 16th row is decoded under a constraint: the second half of the vocabulary is excluded
    x[5::16, vocab // 2:] = -math.inf
    # a trained model: the given token leads by some way in most rows
    x[at, targets] = (torch.rand(rows, generator=gen, device="cuda") * 16).to(dt)
    # some rows carry no token to score
    targets = torch.where(at % 13 == 7, -1, targets)
    st["logits"], st["targets"] = x, targets.to(torch.int32)
    if case["op"] == "logprobs_grad":
        st["g_logprob"] = -torch.rand(rows, generator=gen, device="cuda") / rows
        st["g_entropy"] = torch.randn(rows, generator=gen, device="cuda") * (0.1 / rows) if case["entropy"] else None
    return st


def prepare(case, seed):
    st = _make_inputs(case, seed)
    if case["op"] == "attn_grad":  # what the forward pass has left
        st["out"], st["lse"] = _plain_attention(st)
    if case["op"] == "logprobs_grad":
        _, st["lse"], st["entropy"], _, _ = _plain_logprobs(st, 0)
    if own:
        _prepare_own(st)
    return st


def work(case):
    eb = 4 if case["dtype"] == "f32" else 2
    if case["op"] in SEQUENCE_OPS:
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        prompt, _, attr_len, value_len = _lengths(case)
        n = sum(prompt) + sum(attr_len) + sum(value_len)
        if case["op"] == "rotate":
            return dict(bytes=n * 2 * (hq + hkv) * d * eb, flops=3.0 * n * (hq + hkv) * d)
        pairs = _pairs(case)
        if case["op"] == "attn":
            return dict(bytes=n * ((2 * hq + 2 * hkv) * d * eb + 4 * hq), flops=4.0 * pairs * hq * d)
        return dict(bytes=n * ((4 * hq + 4 * hkv) * d * eb + 4 * hq), flops=10.0 * pairs * hq * d)
    n, v = case["rows"], case["vocab"]
    if case["op"] == "logprobs":  # exp, two sums and a comparison per logit
        return dict(bytes=n * (v * eb + 16 + 8 * case["top"]), flops=6.0 * n * v)
    return dict(bytes=n * (2 * v * eb + 16 + (8 if case["entropy"] else 0)), flops=4.0 * n * v)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(st):
    op = st["case"]["op"]
    if own:
        return _OWN[op](st)
    if op == "rotate":
        return _plain_rotate(st)
    if op == "attn":
        return _plain_attention(st)
    if op == "attn_grad":
        return _plain_attention_grad(st)
    if op == "logprobs":
        return _plain_logprobs(st, st["case"]["top"])
    return _plain_logprobs_grad(st)


def _angles(pos, case):
    d = case["d"]
    theta = case["base"] ** (-torch.arange(0, d, 2, device=pos.device, dtype=torch.float64) / d)
    a = pos[:, None].double() * theta
    return torch.cos(a).float(), torch.sin(a).float()


def _plain_rotate(st):
    """Channel pairs (m, m + d/2) of q and k turned by the token's position ID."""
    case = st["case"]
    cos, sin = _angles(torch.cat([pos for pos, _ in st["seqs"]]), case)
    cos, sin = cos[:, None], (-sin if case["inverse"] else sin)[:, None]
    h, out = case["d"] // 2, []
    for x in (st["q"], st["k"]):
        a, b = x[..., :h].float(), x[..., h:].float()
        out.append(torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1).to(x.dtype))
    return tuple(out)


def _head_groups(case, s):
    """kv heads taken at once: score matrices of about 1 GB at most."""
    g = case["hq"] // case["hkv"]
    per = max(1, min(case["hkv"], int(2.7e8 // max(1, g * s * s))))
    return [(a, min(a + per, case["hkv"])) for a in range(0, case["hkv"], per)]


def _plain_scores(st, a, b, lo, hi, rank):
    """Masked scores of kv heads a..b of one sequence, [b-a, G*S, S], with q and k in 32 bits."""
    case = st["case"]
    g, s, d = case["hq"] // case["hkv"], hi - lo, case["d"]
    q = st["q"][lo:hi, a * g:b * g].float().transpose(0, 1).reshape(b - a, g * s, d)
    k = st["k"][lo:hi, a:b].float().transpose(0, 1)
    scores = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(d)
    at = torch.arange(s, device=rank.device)
    seen = (at[None, :] <= at[:, None]) & (rank[None, :] <= rank[:, None])
    scores = torch.where(seen, scores.view(b - a, g, s, s), -math.inf).view(b - a, g * s, s)
    return q, k, scores


def _plain_attention(st):
    case = st["case"]
    n, hq, d = st["q"].shape
    g = hq // case["hkv"]
    out = torch.empty((n, hq, d), dtype=st["q"].dtype, device=st["q"].device)
    lse = torch.empty((hq, n), dtype=torch.float32, device=st["q"].device)
    lo = 0
    for _, rank in st["seqs"]:
        s = rank.numel()
        hi = lo + s
        if s:
            for a, b in _head_groups(case, s):
                _, _, scores = _plain_scores(st, a, b, lo, hi, rank)
                top = scores.amax(dim=-1, keepdim=True)
                p = torch.exp(scores - top)
                total = p.sum(dim=-1, keepdim=True)
                v = st["v"][lo:hi, a:b].float().transpose(0, 1)
                o = torch.matmul(p, v) / total
                out[lo:hi, a * g:b * g] = o.view((b - a) * g, s, d).transpose(0, 1).to(out.dtype)
                lse[a * g:b * g, lo:hi] = (top + torch.log(total)).view((b - a) * g, s)
        lo = hi
    return out, lse


def _plain_attention_grad(st):
    case = st["case"]
    dt, dev = st["q"].dtype, st["q"].device
    n, hq, d = st["q"].shape
    hkv = case["hkv"]
    g = hq // hkv
    dq = torch.empty((n, hq, d), dtype=dt, device=dev)
    dk = torch.empty((n, hkv, d), dtype=dt, device=dev)
    dv = torch.empty((n, hkv, d), dtype=dt, device=dev)
    lo = 0
    for _, rank in st["seqs"]:
        s = rank.numel()
        hi = lo + s
        if s:
            for a, b in _head_groups(case, s):
                q, k, scores = _plain_scores(st, a, b, lo, hi, rank)
                p = torch.exp(scores - st["lse"][a * g:b * g, lo:hi].reshape(b - a, g * s, 1))
                v = st["v"][lo:hi, a:b].float().transpose(0, 1)
                do = st["d_out"][lo:hi, a * g:b * g].float().transpose(0, 1).reshape(b - a, g * s, d)
                o = st["out"][lo:hi, a * g:b * g].float().transpose(0, 1).reshape(b - a, g * s, d)
                delta = (do * o).sum(dim=-1, keepdim=True)
                dv_ = torch.matmul(p.transpose(1, 2), do)
                ds = p * (torch.matmul(do, v.transpose(1, 2)) - delta) / math.sqrt(d)
                dq_ = torch.matmul(ds, k).view((b - a) * g, s, d)
                dk_ = torch.matmul(ds.transpose(1, 2), q)
                dq[lo:hi, a * g:b * g] = dq_.transpose(0, 1).to(dt)
                dk[lo:hi, a:b] = dk_.transpose(0, 1).to(dt)
                dv[lo:hi, a:b] = dv_.transpose(0, 1).to(dt)
        lo = hi
    return dq, dk, dv


def _plain_logprobs(st, top):
    """Log probability of the row's token (0 where there is none), log of the sum of exponentials,
    entropy, and the ``top`` most likely tokens (lowest index first among equals)."""
    x, t = st["logits"].float(), st["targets"].long()
    m = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(dim=1, keepdim=True)
    lse = (m + torch.log(total))[:, 0]
    diff = torch.where(e > 0, x - m, 0.0)
    entropy = torch.log(total)[:, 0] - (e * diff).sum(dim=1) / total[:, 0]
    valid = (t >= 0) & (t < x.shape[1])
    at = torch.arange(x.shape[0], device=x.device)
    logprob = torch.where(valid, x[at, torch.where(valid, t, 0)] - lse, 0.0)
    column = torch.arange(x.shape[1], device=x.device, dtype=torch.int32)
    ids = torch.empty((x.shape[0], top), dtype=torch.int32, device=x.device)
    vals = torch.empty((x.shape[0], top), dtype=torch.float32, device=x.device)
    left = torch.ones(x.shape, dtype=torch.bool, device=x.device) if top else None
    for i in range(top):
        best = torch.where(left, x, -math.inf).amax(dim=1, keepdim=True)
        at_best = torch.where(left & (x == best), column, 2 ** 31 - 1).amin(dim=1)
        ids[:, i] = at_best
        vals[:, i] = best[:, 0] - lse
        left[at, at_best.long()] = False
    return logprob, lse, entropy, ids, vals


def _plain_logprobs_grad(st):
    x, t = st["logits"].float(), st["targets"].long()
    lp = x - st["lse"][:, None]
    p = torch.exp(lp)
    valid = (t >= 0) & (t < x.shape[1])
    g = torch.where(valid, st["g_logprob"], 0.0)
    dx = -g[:, None] * p
    if st["g_entropy"] is not None:
        dx = dx - torch.where(p > 0, st["g_entropy"][:, None] * p * (lp + st["entropy"][:, None]), 0.0)
    at = torch.arange(x.shape[0], device=x.device)
    dx[at, torch.where(valid, t, 0)] += g
    return dx.to(st["logits"].dtype)


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------
def _prepare_own(st):
    from paper_2604_26209_amd import binding as B

    case = st["case"]
    dt = B.HPD_F32 if case["dtype"] == "f32" else B.HPD_BF16
    st["B"], st["dt"] = B, dt
    if case["op"] in SEQUENCE_OPS:
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        prompt, attr_ptr, attr_len, value_len = _lengths(case)
        cfg = B.hpd_finetune_config(hq, hkv, d, dt, case["base"], case["k_max"], 0)
        st["layout"] = B.hpd_build_finetune_layout(cfg, prompt, attr_ptr, attr_len, value_len)
        n = st["q"].shape[0]

        def empty(shape):
            return torch.empty(shape, dtype=_dtype(case), device="cuda")

        if case["op"] == "rotate":  # gradients go back into the layout of what they belong to
            st["q_out"], st["k_out"], _ = _qkv_buffers(dict(case, fused=case["fused"] and case["inverse"]), n, empty)
            st["strides"] = B.hpd_finetune_strides(st["q"].stride(0), st["k"].stride(0), 0, st["q_out"].stride(0),
                                                   st["k_out"].stride(0), 0)
            return
        st["workspace"] = B.alloc_finetune_workspace(st["layout"], backward=case["op"] == "attn_grad")
        if case["op"] == "attn":
            st["out"] = empty((n, hq, d))
            st["lse"] = torch.empty((hq, n), dtype=torch.float32, device="cuda")
            st["strides"] = B.hpd_finetune_strides(v=st["v"].stride(0))
        else:
            st["dq"], st["dk"] = empty((n, hq, d)), empty((n, hkv, d))
            st["dv"] = _qkv_buffers(case, n, empty)[2]
            st["strides"] = B.hpd_finetune_strides(v=st["v"].stride(0), v_out=st["dv"].stride(0))
        return
    rows, vocab = case["rows"], case["vocab"]
    if case["op"] == "logprobs":
        st["workspace"] = torch.empty(max(1, B.hpd_token_logprobs_workspace(dt, rows, vocab, case["top"])),
                                      dtype=torch.uint8, device="cuda")
        st["outs"] = [torch.empty(rows, dtype=torch.float32, device="cuda") for _ in range(3)] + [
            torch.empty((rows, case["top"]), dtype=torch.int32, device="cuda"),
            torch.empty((rows, case["top"]), dtype=torch.float32, device="cuda")]
    else:
        st["d_logits"] = torch.empty((rows, vocab), dtype=_dtype(case), device="cuda")


def _own_rotate(st):
    st["B"].hpd_finetune_rotate(st["layout"], st["case"]["inverse"], st["q"], st["k"], st["q_out"], st["k_out"],
                                st["strides"])
    return st["q_out"], st["k_out"]


def _own_attention(st):
    st["B"].hpd_finetune_attention(st["layout"], st["q"], st["k"], st["v"], st["out"], st["lse"], st["workspace"],
                                   st["strides"])
    return st["out"], st["lse"]


def _own_attention_grad(st):
    st["B"].hpd_finetune_attention_backward(st["layout"], st["q"], st["k"], st["v"], st["out"], st["lse"],
                                            st["d_out"], st["dq"], st["dk"], st["dv"], st["workspace"], st["strides"])
    return st["dq"], st["dk"], st["dv"]


def _own_logprobs(st):
    case = st["case"]
    logprob, lse, entropy, ids, vals = st["outs"]
    st["B"].hpd_token_logprobs(st["dt"], case["rows"], case["vocab"], case["stride"], st["logits"], st["targets"],
                               case["top"], logprob, lse, entropy, ids, vals, st["workspace"])
    return logprob, lse, entropy, ids, vals


def _own_logprobs_grad(st):
    case = st["case"]
    st["B"].hpd_token_logprobs_backward(st["dt"], case["rows"], case["vocab"], case["stride"], st["logits"],
                                        st["targets"], st["lse"], st["entropy"], st["g_logprob"], st["g_entropy"],
                                        st["d_logits"], case["vocab"])
    return st["d_logits"]


_OWN = dict(rotate=_own_rotate, attn=_own_attention, attn_grad=_own_attention_grad, logprobs=_own_logprobs,
            logprobs_grad=_own_logprobs_grad)


# ---------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _exact_turn(x, pos, base):
    """x [tokens, d] as d/2 complex numbers, turned by pos * base^(-2m/d)."""
    h = x.shape[1] // 2
    m = torch.arange(h, device=x.device, dtype=torch.float64)
    angle = torch.outer(pos.double(), torch.exp(m * (-math.log(base) / h)))
    z = torch.complex(x[:, :h].double(), x[:, h:].double()) * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], dim=1)


def exact(case, seed):
    st = _make_inputs(case, seed)
    if case["op"] == "rotate":
        pos = torch.cat([p for p, _ in st["seqs"]]) * (-1 if case["inverse"] else 1)
        return tuple(torch.stack([_exact_turn(x[:, h], pos, case["base"]) for h in range(x.shape[1])], dim=1)
                     for x in (st["q"], st["k"]))
    if case["op"] in ("attn", "attn_grad"):
        n, hq, d = st["q"].shape
        hkv = case["hkv"]
        dev = st["q"].device
        grad = case["op"] == "attn_grad"
        out = torch.zeros((n, hq, d), dtype=torch.float64, device=dev)
        lse = torch.zeros((hq, n), dtype=torch.float64, device=dev)
        dq = torch.zeros((n, hq, d), dtype=torch.float64, device=dev)
        dk = torch.zeros((n, hkv, d), dtype=torch.float64, device=dev)
        dv = torch.zeros((n, hkv, d), dtype=torch.float64, device=dev)
        start = 0
        for pos, rank in st["seqs"]:
            sl = slice(start, start + pos.numel())
            start += pos.numel()
            if pos.numel() == 0:
                continue
            hidden = torch.triu(torch.ones(pos.numel(), pos.numel(), dtype=torch.bool, device=dev), 1)
            hidden |= rank.unsqueeze(0) > rank.unsqueeze(1)
            for h in range(hq):
                c = h // (hq // hkv)
                qh, kh = st["q"][sl, h].double() / math.sqrt(d), st["k"][sl, c].double()
                vh = st["v"][sl, c].double()
                logits = (qh @ kh.T).masked_fill_(hidden, -math.inf)
                norm = torch.logsumexp(logits, dim=1)
                prob = logits.sub_(norm[:, None]).exp_()
                oh = prob @ vh
                out[sl, h], lse[h, sl] = oh, norm
                if grad:
                    gh = st["d_out"][sl, h].double()
                    dv[sl, c] += prob.T @ gh
                    prob *= gh @ vh.T - (gh * oh).sum(dim=1, keepdim=True)
                    dq[sl, h] = prob @ kh / math.sqrt(d)
                    dk[sl, c] += prob.T @ qh
        return (dq, dk, dv) if grad else (out, lse)
    logits, targets = st["logits"], st["targets"].long()
    parts = []
    for a in range(0, case["rows"], 256):
        x = logits[a:a + 256].double()
        t = targets[a:a + 256]
        lse = torch.logsumexp(x, dim=1)
        lp = x - lse[:, None]
        prob = lp.exp()
        entropy = -torch.special.xlogy(prob, prob).sum(dim=1)
        rows = torch.nonzero(t >= 0)[:, 0]
        if case["op"] == "logprobs":
            logprob = torch.zeros_like(lse)
            logprob[rows] = lp[rows, t[rows]]
            vals, ids = torch.sort(logits[a:a + 256], dim=1, descending=True, stable=True)
            ids = ids[:, :case["top"]]
            parts.append((logprob, lse, entropy, ids.to(torch.int32), torch.gather(lp, 1, ids)))
        else:
            g = torch.where(t >= 0, st["g_logprob"][a:a + 256].double(), 0.0)
            dx = -g[:, None] * prob
            if st["g_entropy"] is not None:
                finite = torch.where(prob > 0, lp, 0.0)
                dx -= st["g_entropy"][a:a + 256].double()[:, None] * prob * (finite + entropy[:, None])
            dx[rows, t[rows]] += g[rows]
            parts.append((dx,))
    joined = tuple(torch.cat(p) for p in zip(*parts))
    return joined if case["op"] == "logprobs" else joined[0]
