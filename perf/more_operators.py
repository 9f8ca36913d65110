"""The two ends of a fine-tuned layer stack as cases to be measured: the gated feed-forward block and the
vocabulary head with the log probabilities of given tokens, each with its gradient.

    feed-forward   out = (act(x Wg^T) * (x Wu^T)) Wd^T; a training step keeps x Wg^T and x Wu^T
    head           log probability of the row's token, log of the sum of exponentials and entropy of
                   softmax(hidden W^T), without the logits in memory

``run`` computes them in elementary torch operations where ``own`` is false and through the library
where it is true.

Sizes: widths are heads x channels of the benchmark's configurations and of the tests, inner widths two
to four times that, rows those of a decode step (branches) or of a training batch; vocabularies are generic.
"""
import math

import torch

own = False

# the largest cases that are drawn: operations, bytes read and written
BF16_FLOPS, F32_FLOPS, BYTES = 6.5e12, 4e11, 2.2e9
WIDTHS = [256, 480, 512, 1152, 2048, 4096, 4096, 5120, 8192]  # heads x channels
ACTS = ["silu", "silu", "gelu", "gelu_tanh"]
INPUT_SEED, PIECE = 977, 1 << 15


def listed():
    return [
        # one token: the last branch of a decode step
        dict(name="ffn_token", op="ffn", dtype="bf16", rows=1, width=4096, inner=12288, act="silu", keep=False, fused=True),
        # the live branches of a decode step of 32 prompts with 16 attributes each
        dict(name="ffn_decode", op="ffn", dtype="bf16", rows=512, width=4096, inner=12288, act="silu", keep=False, fused=True),
        # a training batch of stacked documents, ragged
        dict(name="ffn_batch", op="ffn", dtype="bf16", rows=14903, width=4096, inner=12288, act="silu", keep=True, fused=True),
        # the small fp32 layer, the smallest call
        dict(name="ffn_f32_small", op="ffn", dtype="f32", rows=333, width=256, inner=1000, act="gelu", keep=True, fused=False),
        # gradients of a training batch of single documents
        dict(name="ffn_grad_batch", op="ffn_grad", dtype="bf16", rows=8191, width=4096, inner=12288, act="silu", weights=True,
             fused=True),
        # ... of a short sequence with frozen weights, as under adapters
        dict(name="ffn_grad_frozen", op="ffn_grad", dtype="bf16", rows=190, width=2048, inner=5504, act="gelu_tanh",
             weights=False, fused=False),
        # ... in fp32
        dict(name="ffn_grad_f32", op="ffn_grad", dtype="f32", rows=1801, width=1152, inner=4008, act="gelu", weights=True,
             fused=False),
        # the value tokens of a training batch over a large vocabulary
        dict(name="head_batch", op="head", dtype="bf16", rows=6144, width=4096, vocab=130013),
        # three tokens scored while decoding
        dict(name="head_few", op="head", dtype="bf16", rows=3, width=4096, vocab=150001),
        # the loss' gradient over the value tokens of a batch, smaller vocabulary
        dict(name="head_grad_batch", op="head_grad", dtype="bf16", rows=4096, width=4096, vocab=32000, entropy=False,
             weights=True),
        # with an entropy term, a large vocabulary
        dict(name="head_grad_wide", op="head_grad", dtype="bf16", rows=2021, width=4096, vocab=130013, entropy=True,
             weights=True),
        # fp32, frozen head
        dict(name="head_grad_f32", op="head_grad", dtype="f32", rows=700, width=1152, vocab=50021, entropy=True,
             weights=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["ffn", "ffn", "ffn_grad", "head", "head_grad"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    while True:
        case = dict(op=op, dtype=dtype, rows=_log_int(rng, 1, 20000), width=rng.choice(WIDTHS))
        if op in ("ffn", "ffn_grad"):
            case["inner"] = 8 * rng.randint(case["width"] // 4, case["width"] // 2)
            case["act"], case["fused"] = rng.choice(ACTS), rng.random() < 0.5
        else:
            case["vocab"] = _log_int(rng, 200, 160000)
        if op == "ffn":
            case["keep"] = rng.random() < 0.5
        if op == "head_grad":
            case["entropy"] = rng.random() < 0.5
        if op.endswith("grad"):
            case["weights"] = rng.random() < 0.7
        w = work(case)
        if w["flops"] <= (BF16_FLOPS if dtype == "bf16" else F32_FLOPS) and w["bytes"] <= BYTES:
            return case


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def work(case):
    eb, n, d = 4 if case["dtype"] == "f32" else 2, case["rows"], case["width"]
    if case["op"] == "ffn":
        f = case["inner"]
        return dict(bytes=eb * (2 * n * d + 3 * d * f + (2 * n * f if case["keep"] else 0)), flops=6.0 * n * d * f)
    if case["op"] == "ffn_grad":
        f = case["inner"]
        rows = 2 * n * d + 2 * n * f  # d_out, gate, up read, d_x written
        if case["weights"]:
            return dict(bytes=eb * (rows + n * d + 6 * d * f), flops=12.0 * n * d * f)
        return dict(bytes=eb * (rows + 3 * d * f), flops=6.0 * n * d * f)
    v = case["vocab"]
    if case["op"] == "head":
        return dict(bytes=eb * (n * d + v * d) + 16 * n, flops=2.0 * n * d * v)
    out = n * d + (v * d if case["weights"] else 0)
    return dict(bytes=eb * (n * d + v * d + out) + (20 if case["entropy"] else 12) * n,
                flops=(6.0 if case["weights"] else 4.0) * n * d * v)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _make_inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(INPUT_SEED + int(seed))
    dt, n, d = _dtype(case), case["rows"], case["width"]

    def normal(rows, cols, std=1.0):
        out = torch.empty((rows, cols), dtype=dt, device="cuda")
        for a in range(0, rows, PIECE):
            b = min(a + PIECE, rows)
            out[a:b] = (torch.randn((b - a, cols), generator=gen, device="cuda") * std).to(dt)
        return out

    st = dict(case=case)
    if case["op"] in ("ffn", "ffn_grad"):
        f = case["inner"]
        st["x"] = normal(n, d)  # a normalised residual stream
        w = normal(2 * f, d, d ** -0.5)
        # one matrix for both projections, or two
        st["w_gate"], st["w_up"] = (w[:f], w[f:]) if case["fused"] else (w[:f].clone(), w[f:].clone())
        st["w_down"] = normal(d, f, f ** -0.5)
        if case["op"] == "ffn_grad":  # what the forward pass has kept
            kept = torch.empty((n, 2 * f) if case["fused"] else (2, n, f), dtype=dt, device="cuda")
            st["gate"], st["up"] = (kept[:, :f], kept[:, f:]) if case["fused"] else (kept[0], kept[1])
            x = st["x"].float()
            st["gate"].copy_(torch.matmul(x, st["w_gate"].float().t()))
            st["up"].copy_(torch.matmul(x, st["w_up"].float().t()))
            st["d_out"] = normal(n, d, 1.0 / n)
        return st
    v = case["vocab"]
    st["weight"] = normal(v, d, 2.5 * d ** -0.5)  # logits of a standard deviation of 2.5
    targets = torch.randint(0, v, (n,), generator=gen, device="cuda")
    # a trained model: the given token leads by some way in most rows
    lead = torch.rand((n, 1), generator=gen, device="cuda") * (16 / 6.25)
    st["hidden"] = (torch.randn((n, d), generator=gen, device="cuda") + lead * st["weight"][targets].float()).to(dt)
    # some rows carry no token to score
    st["targets"] = torch.where(torch.arange(n, device="cuda") % 13 == 7, -1, targets).to(torch.int32)
    if case["op"] == "head_grad":
        st["g_logprob"] = -torch.rand(n, generator=gen, device="cuda") / n
        st["g_entropy"] = torch.randn(n, generator=gen, device="cuda") * (0.1 / n) if case["entropy"] else None
    return st


def prepare(case, seed):
    st = _make_inputs(case, seed)
    if case["op"] == "head_grad":  # what the forward pass has left
        _, st["lse"], st["entropy"] = _plain_head(st)
    if own:
        _prepare_own(st)
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(st):
    op = st["case"]["op"]
    if own:
        return _OWN[op](st)
    return dict(ffn=_plain_ffn, ffn_grad=_plain_ffn_grad, head=_plain_head, head_grad=_plain_head_grad)[op](st)


def _plain_act(a, act):
    """The activation and its derivative."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-a))
        return a * s, s * (1 + a * (1 - s))
    if act == "gelu":
        c = 0.5 * (1 + torch.erf(a * math.sqrt(0.5)))
        return a * c, c + a * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (a + 0.044715 * a * a * a))
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * k * (1 + 3 * 0.044715 * a * a)


def _plain_ffn(st):
    case, dt = st["case"], st["x"].dtype
    x = st["x"].float()
    gate = torch.matmul(x, st["w_gate"].float().t())
    up = torch.matmul(x, st["w_up"].float().t())
    h = _plain_act(gate, case["act"])[0] * up
    out = torch.matmul(h, st["w_down"].float().t()).to(dt)
    return (out, gate.to(dt), up.to(dt)) if case["keep"] else out


def _plain_ffn_grad(st):
    case, dt = st["case"], st["x"].dtype
    gate, up, d_out = st["gate"].float(), st["up"].float(), st["d_out"].float()
    act, slope = _plain_act(gate, case["act"])
    d_h = torch.matmul(d_out, st["w_down"].float())
    d_gate, d_up = d_h * up * slope, d_h * act
    d_x = (torch.matmul(d_gate, st["w_gate"].float()) + torch.matmul(d_up, st["w_up"].float())).to(dt)
    if not case["weights"]:
        return d_x
    x = st["x"].float()
    return (d_x, torch.matmul(d_gate.t(), x).to(dt), torch.matmul(d_up.t(), x).to(dt),
            torch.matmul(d_out.t(), act * up).to(dt))


def _plain_head(st):
    x, w, t = st["hidden"].float(), st["weight"], st["targets"].long()
    n, v = x.shape[0], w.shape[0]
    logits = torch.empty((n, v), dtype=torch.float32, device=x.device)
    for a in range(0, v, PIECE):
        b = min(a + PIECE, v)
        logits[:, a:b] = torch.matmul(x, w[a:b].float().t())
    valid = (t >= 0) & (t < v)
    of_target = logits[torch.arange(n, device=x.device), torch.where(valid, t, 0)]
    m = logits.amax(dim=1, keepdim=True)
    logits -= m
    e = torch.exp(logits)
    total = e.sum(dim=1)
    mean = e.mul_(logits).sum(dim=1) / total
    lse = m[:, 0] + torch.log(total)
    return torch.where(valid, of_target - lse, 0.0), lse, torch.log(total) - mean


def _plain_head_grad(st):
    case, x, w, t = st["case"], st["hidden"].float(), st["weight"], st["targets"].long()
    n, v = x.shape[0], w.shape[0]
    valid = (t >= 0) & (t < v)
    g = torch.where(valid, st["g_logprob"], 0.0)[:, None]
    d_hidden = torch.zeros_like(x)
    d_weight = torch.empty_like(w) if case["weights"] else None
    column = torch.arange(v, device=x.device)
    for a in range(0, v, PIECE):
        b = min(a + PIECE, v)
        piece = w[a:b].float()
        lp = torch.matmul(x, piece.t()) - st["lse"][:, None]
        p = torch.exp(lp)
        dl = torch.where(column[None, a:b] == t[:, None], g, 0.0) - g * p
        if st["g_entropy"] is not None:
            dl -= st["g_entropy"][:, None] * p * (lp + st["entropy"][:, None])
        d_hidden += torch.matmul(dl, piece)
        if case["weights"]:
            d_weight[a:b] = torch.matmul(dl.t(), x).to(w.dtype)
    d_hidden = d_hidden.to(st["hidden"].dtype)
    return (d_hidden, d_weight) if case["weights"] else d_hidden


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------
def _prepare_own(st):
    from paper_2604_26209_amd import binding as B

    case = st["case"]
    dt, td, n, d = B.HPD_F32 if case["dtype"] == "f32" else B.HPD_BF16, _dtype(case), case["rows"], case["width"]
    st["B"], st["dt"] = B, dt

    def empty(*shape, t=td):
        return torch.empty(shape, dtype=t, device="cuda")

    if case["op"] in ("ffn", "ffn_grad"):
        f = case["inner"]
        act = dict(silu=B.HPD_ACT_SILU, gelu=B.HPD_ACT_GELU, gelu_tanh=B.HPD_ACT_GELU_TANH)[case["act"]]
        st["cfg"] = B.hpd_ffn_config(d, f, dt, act)
        backward = case["op"] == "ffn_grad"
        st["workspace"] = B.alloc_ffn_workspace(st["cfg"], n, backward=backward)
        if not backward:
            st["out"] = empty(n, d)
            if case["keep"]:
                kept = empty(n, 2 * f) if case["fused"] else empty(2, n, f)
                st["gate"], st["up"] = (kept[:, :f], kept[:, f:]) if case["fused"] else (kept[0], kept[1])
            st["strides"] = B.hpd_ffn_strides(gate=st["gate"].stride(0), up=st["up"].stride(0)) if case["keep"] else None
            return
        st["strides"] = B.hpd_ffn_strides(gate=st["gate"].stride(0), up=st["up"].stride(0))
        st["d_x"] = empty(n, d)
        if case["weights"]:
            w = empty(2 * f, d)
            st["d_w_gate"], st["d_w_up"], st["d_w_down"] = w[:f], w[f:], empty(d, f)
        return
    v = case["vocab"]
    backward = case["op"] == "head_grad"
    st["workspace"] = B.alloc_head_workspace(dt, n, d, v, backward=backward)
    if backward:
        st["d_hidden"] = empty(n, d)
        st["d_weight"] = empty(v, d) if case["weights"] else None
    else:
        st["outs"] = [empty(n, t=torch.float32) for _ in range(3)]


def _own_ffn(st):
    keep = st["case"]["keep"]
    st["B"].hpd_gated_ffn(st["cfg"], st["case"]["rows"], st["x"], st["w_gate"], st["w_up"], st["w_down"], st["out"],
                          st["gate"] if keep else None, st["up"] if keep else None, st["workspace"], st["strides"])
    return (st["out"], st["gate"], st["up"]) if keep else st["out"]


def _own_ffn_grad(st):
    weights = st["case"]["weights"]
    grads = (st["d_w_gate"], st["d_w_up"], st["d_w_down"]) if weights else (None, None, None)
    st["B"].hpd_gated_ffn_backward(st["cfg"], st["case"]["rows"], st["x"], st["w_gate"], st["w_up"], st["w_down"],
                                   st["gate"], st["up"], st["d_out"], st["d_x"], *grads, st["workspace"], st["strides"])
    return (st["d_x"],) + grads if weights else st["d_x"]


def _own_head(st):
    case = st["case"]
    st["B"].hpd_head_logprobs(st["dt"], case["rows"], case["width"], case["vocab"], st["hidden"], case["width"],
                              st["weight"], case["width"], st["targets"], *st["outs"], st["workspace"])
    return tuple(st["outs"])


def _own_head_grad(st):
    case = st["case"]
    st["B"].hpd_head_logprobs_backward(st["dt"], case["rows"], case["width"], case["vocab"], st["hidden"], case["width"],
                                       st["weight"], case["width"], st["targets"], st["lse"], st["entropy"],
                                       st["g_logprob"], st["g_entropy"], st["d_hidden"], case["width"], st["d_weight"],
                                       case["width"], st["workspace"])
    return (st["d_hidden"], st["d_weight"]) if case["weights"] else st["d_hidden"]


_OWN = dict(ffn=_own_ffn, ffn_grad=_own_ffn_grad, head=_own_head, head_grad=_own_head_grad)


# ---------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _exact_hidden(gate, up, act):
    if act == "silu":
        return torch.nn.functional.silu(gate) * up
    return torch.nn.functional.gelu(gate, approximate="tanh" if act == "gelu_tanh" else "none") * up


def exact(case, seed):
    st = _make_inputs(case, seed)
    if case["op"] == "ffn":
        x = st["x"].double()
        gate, up = x @ st["w_gate"].double().T, x @ st["w_up"].double().T
        out = _exact_hidden(gate, up, case["act"]) @ st["w_down"].double().T
        return (out, gate, up) if case["keep"] else out
    if case["op"] == "ffn_grad":
        gate, up = st["gate"].double().requires_grad_(), st["up"].double().requires_grad_()
        h = _exact_hidden(gate, up, case["act"])
        d_out = st["d_out"].double()
        d_gate, d_up = torch.autograd.grad(h, (gate, up), d_out @ st["w_down"].double())
        d_x = d_gate @ st["w_gate"].double() + d_up @ st["w_up"].double()
        if not case["weights"]:
            return d_x
        x = st["x"].double()
        return d_x, d_gate.T @ x, d_up.T @ x, d_out.T @ h.detach()
    n, d, v = case["rows"], case["width"], case["vocab"]
    grad = case["op"] == "head_grad"
    d_weight = torch.zeros((v, d), dtype=torch.float64, device="cuda") if grad and case["weights"] else None
    weight, parts = st["weight"].double(), []
    for a in range(0, n, 1024):
        x, t = st["hidden"][a:a + 1024].double(), st["targets"][a:a + 1024].long()
        rows = torch.nonzero(t >= 0)[:, 0]
        logits = x @ weight.T
        lse = torch.logsumexp(logits, dim=1)
        lp = logits - lse[:, None]
        entropy = -torch.special.xlogy(lp.exp(), lp.exp()).sum(dim=1)
        if not grad:
            logprob = torch.zeros(x.shape[0], dtype=torch.float64, device="cuda")
            logprob[rows] = lp[rows, t[rows]]
            parts.append((logprob, lse, entropy))
            continue
        g = st["g_logprob"][a:a + 1024].double()
        dl = torch.zeros_like(lp)
        dl[rows, t[rows]] = g[rows]
        g = torch.where(t >= 0, g, 0.0)
        if st["g_entropy"] is not None:
            g = g[:, None] + st["g_entropy"][a:a + 1024].double()[:, None] * (lp + entropy[:, None])
        else:
            g = g[:, None]
        dl -= g * lp.exp()
        parts.append((dl @ weight,))
        if d_weight is not None:
            d_weight += dl.T @ x
    joined = tuple(torch.cat(p) for p in zip(*parts))
    if not grad:
        return joined
    return (joined[0], d_weight) if case["weights"] else joined[0]
