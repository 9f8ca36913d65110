"""Log probabilities from hidden states and the vocabulary's weights through the library, and their gradients, against the
definitions in 64 bits."""
import math

import pytest
import torch

import ffn_ref as R
from paper_2604_26209_amd import binding as B
from test_gpu_ffn import DT, TD, Padded

pytestmark = pytest.mark.gpu

SIZES = [(1, 8, 1), (1, 64, 7), (3, 72, 129), (33, 136, 1000), (64, 256, 4099), (65, 64, 127), (130, 480, 1025), (257, 512, 128),
         (300, 128, 2051)]


def _inputs(rows, width, vocab, dtype, seed=0, scale=2.5):
    gen = torch.Generator().manual_seed(seed)
    w = (torch.randn((vocab, width), generator=gen) * scale * width ** -0.5).to(TD[dtype])
    t = torch.randint(0, vocab, (rows,), generator=gen, dtype=torch.int32)
    x = torch.randn((rows, width), generator=gen) + torch.rand((rows, 1), generator=gen) * 2 * w[t.long()].float()
    t[5::7] = -1
    t[6::11] = vocab
    g, ge = (torch.randn(rows, generator=gen).cuda() for _ in range(2))
    return dict(x=x.to(TD[dtype]).cuda(), w=w.cuda(), t=t.cuda(), g=g, ge=ge)


def _forward(i, dtype, pad=8):
    (rows, width), vocab = i["x"].shape, i["w"].shape[0]
    x, w = (Padded(*i[k].shape, TD[dtype], i[k], pad) for k in ("x", "w"))
    outs = [torch.full((rows + 2,), 77.0, device="cuda") for _ in range(3)]
    ws = B.alloc_head_workspace(DT[dtype], rows, width, vocab, backward=False)
    B.hpd_head_logprobs(DT[dtype], rows, width, vocab, x.t, x.t.stride(0), w.t, w.t.stride(0), i["t"],
                        *[o[1:rows + 1] for o in outs], ws)
    torch.cuda.synchronize()
    assert all(o[0] == 77.0 and o[-1] == 77.0 for o in outs)
    return [o[1:rows + 1] for o in outs]


def _backward(i, dtype, lse, entropy, g=True, ge=True, hidden=True, weight=True, pad=8):
    (rows, width), vocab = i["x"].shape, i["w"].shape[0]
    x, w = (Padded(*i[k].shape, TD[dtype], i[k], pad) for k in ("x", "w"))
    dx, dw = Padded(rows, width, TD[dtype], pad=pad), Padded(vocab, width, TD[dtype], pad=pad)
    ws = B.alloc_head_workspace(DT[dtype], rows, width, vocab, backward=True)
    if ws is not None:
        ws.fill_(0xff)  # (NaN in both types)
    B.hpd_head_logprobs_backward(DT[dtype], rows, width, vocab, x.t, x.t.stride(0), w.t, w.t.stride(0), i["t"], lse,
                                 entropy if ge else None, i["g"] if g else None, i["ge"] if ge else None,
                                 dx.t if hidden else None, dx.t.stride(0), dw.t if weight else None, dw.t.stride(0), ws)
    torch.cuda.synchronize()
    assert dx.untouched() and dw.untouched()
    assert hidden or bool((dx.buf == 31744.0).all())
    assert weight or bool((dw.buf == 31744.0).all())
    return dx.t, dw.t


def _check(i, dtype, ge=True):
    x, w = i["x"].double(), i["w"].double()
    got = _forward(i, dtype)
    for name, a, want in zip(("logprob", "lse", "entropy"), got, R.head(x, w, i["t"])):
        R.check(a, want, name)
    _, lse, entropy = got
    want = R.head_grad(x, w, i["t"], lse.double(), entropy.double(), i["g"].double(), i["ge"].double() if ge else None, TD[dtype])
    for name, a, b in zip(("d_hidden", "d_weight"), _backward(i, dtype, lse, entropy, ge=ge), want):
        R.check(a, b, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, width, vocab", SIZES)
@pytest.mark.parametrize("ge", [True, False])
def test_head(rows, width, vocab, dtype, ge):
    _check(_inputs(rows, width, vocab, dtype), dtype, ge)


# large vocabularies in several pieces, many rows, few rows
@pytest.mark.parametrize("dtype, rows, width, vocab", [("bf16", 2, 1152, 50021), ("bf16", 700, 256, 130013), ("f32", 300, 136, 50021),
                                                       ("bf16", 3001, 512, 9001), ("bf16", 40, 4096, 12003), ("bf16", 4100, 72, 33000)])
def test_larger(dtype, rows, width, vocab):
    _check(_inputs(rows, width, vocab, dtype, seed=1), dtype)


# tiles of every size in every product, whole and cut contractions
@pytest.mark.parametrize("dtype, rows, width, vocab", [("bf16", 4100, 2048, 9001), ("bf16", 5000, 1032, 20011), ("bf16", 300, 4096, 20011),
                                                       ("f32", 2, 1152, 50021), ("f32", 33, 520, 9001), ("bf16", 32, 2048, 33001)])
def test_tiles_of_every_size(dtype, rows, width, vocab):
    _check(_inputs(rows, width, vocab, dtype, seed=9), dtype)


# 192 x 256 tiles of logits, 64 x 128 of gradients
@pytest.mark.parametrize("dtype, rows, width, vocab", [("bf16", 500, 1032, 24011), ("bf16", 100, 1032, 30001), ("bf16", 100, 2048, 20011),
                                                       ("bf16", 1000, 1032, 12001), ("bf16", 125, 4096, 9001)])
def test_tiles_between(dtype, rows, width, vocab):
    _check(_inputs(rows, width, vocab, dtype, seed=12), dtype)


def _cut(dtype, rows, width, vocab):
    """Whether the forward call's workspace holds parts of the logits."""
    return B.hpd_head_logprobs_workspace(DT[dtype], rows, width, vocab)[0] >= 2 * 4 * rows * vocab


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, width, vocab, ge", [(1, 8192, 1, True), (5, 8192, 67, True), (69, 8192, 1119, False),
                                                    (130, 5120, 385, True), (33, 4104, 4, True), (2, 16384, 2050, True)])
def test_contractions_in_parts(rows, width, vocab, ge, dtype):
    assert _cut(dtype, rows, width, vocab)
    _check(_inputs(rows, width, vocab, dtype, seed=10), dtype, ge)


def test_contractions_in_parts_not_all_wanted():
    rows, width, vocab = 70, 8192, 515
    assert _cut("bf16", rows, width, vocab)
    i = _inputs(rows, width, vocab, "bf16", seed=13)
    _, lse, entropy = _forward(i, "bf16")
    ws, one, two = B.alloc_head_workspace(B.HPD_BF16, rows, width, vocab, False), *torch.zeros((2, rows), device="cuda")
    B.hpd_head_logprobs(B.HPD_BF16, rows, width, vocab, i["x"], 0, i["w"], 0, None, None, one, None, ws)
    B.hpd_head_logprobs(B.HPD_BF16, rows, width, vocab, i["x"], 0, i["w"], 0, None, None, None, two, ws)
    assert torch.equal(one, lse) and torch.equal(two, entropy)
    dx, dw = _backward(i, "bf16", lse, entropy)
    assert torch.equal(_backward(i, "bf16", lse, entropy, weight=False)[0], dx)
    assert torch.equal(_backward(i, "bf16", lse, entropy, hidden=False)[1], dw)


@pytest.mark.parametrize("hidden, weight, g, ge", [(1, 0, 1, 1), (0, 1, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (1, 1, 0, 0)])
def test_parts_that_are_not_wanted(hidden, weight, g, ge):
    i = _inputs(70, 136, 500, "bf16", seed=2)
    _, lse, entropy = _forward(i, "bf16")
    want = R.head_grad(i["x"].double(), i["w"].double(), i["t"], lse.double(), entropy.double(), i["g"].double() if g else None,
                       i["ge"].double() if ge else None, torch.bfloat16)
    dx, dw = _backward(i, "bf16", lse, entropy, g, ge, hidden, weight)
    if hidden:
        R.check(dx, want[0], "d_hidden")
    if weight:
        R.check(dw, want[1], "d_weight")


def test_outputs_that_are_not_wanted():
    i = _inputs(70, 136, 500, "bf16", seed=3)
    want = _forward(i, "bf16")
    rows, width, vocab = 70, 136, 500
    ws = B.alloc_head_workspace(B.HPD_BF16, rows, width, vocab, backward=False)
    for n in range(3):
        outs = [torch.empty(rows, device="cuda") if k == n else None for k in range(3)]
        B.hpd_head_logprobs(B.HPD_BF16, rows, width, vocab, i["x"], width, i["w"], width, i["t"], *outs, ws)
        assert torch.equal(outs[n], want[n])
    lse = torch.empty(rows, device="cuda")
    untouched = torch.full((rows,), 5.0, device="cuda")
    B.hpd_head_logprobs(B.HPD_BF16, rows, width, vocab, i["x"], width, i["w"], width, None, untouched, lse, None, ws)
    assert torch.equal(lse, want[1]) and bool((untouched == 5.0).all())


def test_no_rows():
    i = _inputs(0, 64, 40, "bf16")
    _forward(i, "bf16")
    none = torch.empty(1, device="cuda")
    dx, dw = _backward(i, "bf16", none, none)
    assert bool((dw == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 150])
def test_rows_that_are_not_finite(rows, dtype):
    _check_not_finite(rows, 72, 300, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_are_not_finite_in_parts(dtype):
    assert _cut(dtype, 5, 8192, 300) and _cut(dtype, 5, 8192, 1)
    _check_not_finite(5, 8192, 300, dtype)


def _check_not_finite(rows, width, vocab, dtype):
    """+infinity and NaN among a row's logits: NaN in that row alone.  -infinity: a token of probability 0."""
    i = _inputs(rows, width, vocab, dtype, seed=4)
    i["t"][3] = 7
    i["x"][:, 0] = 1.0
    i["w"][:, 0] = 0.0
    clean = [t.clone() for t in _forward(i, dtype)]
    keep = torch.arange(rows, device="cuda") != 3
    for bad in (float("nan"), float("inf")):
        j = dict(i, x=i["x"].clone())
        j["x"][3, 5] = bad
        got = _forward(j, dtype)
        for a, b in zip(got, clean):
            assert torch.equal(a[keep], b[keep]) and bool(torch.isnan(a[3]))
        dx, dw = _backward(j, dtype, got[1], got[2])
        ref, _ = _backward(i, dtype, clean[1], clean[2])
        assert torch.equal(dx[keep], ref[keep]) and bool(torch.isnan(dx[3]).all())
    # an excluded token: its weights times a channel that is 1 in every row give -infinity
    j = dict(i, w=i["w"].clone())
    j["w"][17, 0] = float("-inf")
    j["t"][2] = 17
    logits = j["x"].double() @ i["w"].double().T
    logits[:, 17] = float("-inf")
    got = _forward(j, dtype)
    e = width * R.U * (j["x"].double().abs() @ i["w"].double().abs().T)
    for name, a, want in zip(("logprob", "lse", "entropy"), got, R.logprobs(logits, j["t"], e)):
        value, bound = want
        gone = torch.isinf(value)
        assert torch.equal(a.double()[gone], value[gone])
        R.check(a[~gone], (value[~gone], bound[~gone]), name)
    # rows of nothing else
    j["w"] = j["w"][17:18].clone()
    j["t"] = torch.zeros_like(j["t"])
    logprob, lse, entropy = _forward(j, dtype)
    assert bool((lse == float("-inf")).all() and (logprob == float("-inf")).all() and (entropy == 0).all())


@pytest.mark.parametrize("scale", [1e-3, 100.0, 3e4, 1e15])
def test_logits_of_any_size(scale):
    i = _inputs(40, 64, 700, "f32", seed=5, scale=scale)
    for name, a, want in zip(("logprob", "lse", "entropy"), _forward(i, "f32"), R.head(i["x"].double(), i["w"].double(), i["t"])):
        R.check(a, want, name)


@pytest.mark.parametrize("rows", [3, 200])
def test_equal_calls_give_equal_bits_on_any_stream_and_in_a_graph(rows):
    _check_equal_bits(rows, 264, 5003)


def test_equal_calls_give_equal_bits_in_parts():
    assert _cut("bf16", 70, 8192, 515)
    _check_equal_bits(70, 8192, 515)


def _check_equal_bits(rows, width, vocab):
    i = _inputs(rows, width, vocab, "bf16", seed=6)
    outs = [torch.empty(rows, device="cuda") for _ in range(3)]
    dx, dw = torch.empty_like(i["x"]), torch.empty_like(i["w"])
    ws = [B.alloc_head_workspace(B.HPD_BF16, rows, width, vocab, b) for b in (False, True)]

    def step():
        B.hpd_head_logprobs(B.HPD_BF16, rows, width, vocab, i["x"], width, i["w"], width, i["t"], *outs, ws[0])
        B.hpd_head_logprobs_backward(B.HPD_BF16, rows, width, vocab, i["x"], width, i["w"], width, i["t"], outs[1], outs[2], i["g"],
                                     i["ge"], dx, width, dw, width, ws[1])

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (*outs, dx, dw)]

    def forget():
        for t in (*outs, dx, dw):
            t.fill_(float("nan"))

    step()
    want = results()
    forget()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(results(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x = i["x"].clone()
    for n in range(4):
        forget()
        i["x"].copy_(x if n % 2 == 0 else x * 0.5)
        graph.replay()
        got = results()
        forget()
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, results())), n


def test_the_same_as_from_stored_logits():
    """hpd_token_logprobs on logits in fp32 gives the same numbers."""
    i = _inputs(50, 136, 3001, "f32", seed=7)
    got = _forward(i, "f32")
    logits = (i["x"].double() @ i["w"].double().T).float()
    outs = [torch.empty(50, device="cuda") for _ in range(3)]
    ws = torch.empty(max(1, B.hpd_token_logprobs_workspace(B.HPD_F32, 50, 3001, 0)), dtype=torch.uint8, device="cuda")
    B.hpd_token_logprobs(B.HPD_F32, 50, 3001, 3001, logits, i["t"], 0, *outs, None, None, ws)
    # both within the bound of the definition
    for a, b, (_, bound) in zip(got, outs, R.head(i["x"].double(), i["w"].double(), i["t"])):
        assert bool(((a.double() - b.double()).abs() <= 2 * bound + 1e-37).all())


def test_weights_behind_4_gb():
    """Rows of weights further than 2^32 bytes from the first, in pieces and at once."""
    rows, width, vocab = 4, 16384, 140001
    gen = torch.Generator(device="cuda").manual_seed(8)
    w = torch.zeros((vocab, width), dtype=torch.bfloat16, device="cuda")
    far = torch.tensor([0, 1, 70000, 131071, 131072, 131073, 139999, 140000], device="cuda")
    w[far] = (torch.randn((8, width), generator=gen, device="cuda") * width ** -0.5).bfloat16()
    x = torch.randn((rows, width), generator=gen, device="cuda").bfloat16()
    t = torch.tensor([140000, 131072, 3, 0], dtype=torch.int32, device="cuda")
    outs = [torch.empty(rows, device="cuda") for _ in range(3)]
    ws = B.alloc_head_workspace(B.HPD_BF16, rows, width, vocab, False)
    B.hpd_head_logprobs(B.HPD_BF16, rows, width, vocab, x, width, w, width, t, *outs, ws)
    logits = torch.zeros((rows, vocab), dtype=torch.float64, device="cuda")
    logits[:, far] = x.double() @ w[far].double().T
    e = torch.zeros_like(logits)
    e[:, far] = width * R.U * (x.double().abs() @ w[far].double().abs().T)
    for name, a, want in zip(("logprob", "lse", "entropy"), outs, R.logprobs(logits, t, e)):
        R.check(a, want, name)
    g = torch.ones(rows, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = B.alloc_head_workspace(B.HPD_BF16, rows, width, vocab, True)
    B.hpd_head_logprobs_backward(B.HPD_BF16, rows, width, vocab, x, width, w, width, t, outs[1], None, g, None, dx, width, dw, width, ws)
    p = torch.exp(logits - outs[1].double()[:, None])
    d = -p
    d[torch.arange(rows, device="cuda"), t.long()] += 1
    want = d[:, far] @ w[far].double()
    assert bool(((dx.double() - want).abs() <= 2.0 ** -7 * (d[:, far].abs() @ w[far].double().abs()) + 1e-30).all())
    want = d[:, far].T @ x.double()
    assert bool(((dw[far].double() - want).abs() <= 2.0 ** -6 * (d[:, far].abs().T @ x.double().abs())).all())


@pytest.mark.parametrize("dtype, rows, width, vocab", [("bf16", 600, 256, 9001), ("f32", 300, 264, 501), ("bf16", 520, 4096, 33)])
def test_rows_8_mb_apart(dtype, rows, width, vocab):
    """The widest strides of hidden states and their gradients: the bits of rows without gaps."""
    i = _inputs(rows, width, vocab, dtype, seed=11)
    stride = (8 << 20) // i["x"].element_size()
    far = torch.empty((rows, stride), dtype=TD[dtype], device="cuda")
    x, dx = far[:, :width], far[:, width:2 * width]
    x.copy_(i["x"])
    ws = [B.alloc_head_workspace(DT[dtype], rows, width, vocab, b) for b in (False, True)]

    def run(x, x_stride, dx):
        outs, dw = [torch.empty(rows, device="cuda") for _ in range(3)], torch.empty_like(i["w"])
        B.hpd_head_logprobs(DT[dtype], rows, width, vocab, x, x_stride, i["w"], 0, i["t"], *outs, ws[0])
        B.hpd_head_logprobs_backward(DT[dtype], rows, width, vocab, x, x_stride, i["w"], 0, i["t"], outs[1], outs[2], i["g"], i["ge"],
                                     dx, x_stride, dw, 0, ws[1])
        return (*outs, dx, dw)

    for a, b in zip(run(x, stride, dx), run(i["x"], 0, torch.empty_like(i["x"]))):
        assert torch.equal(a, b)


# sizes for which a plan of each call's own would sum the logits in another order
@pytest.mark.parametrize("dtype, rows, width, vocab", [("f32", 117, 480, 2057), ("f32", 231, 1152, 2057), ("f32", 4, 480, 1100),
                                                       ("f32", 14, 1152, 10404), ("f32", 40, 480, 2057), ("f32", 17, 2048, 23311),
                                                       ("bf16", 6, 2048, 4037), ("bf16", 20, 2048, 6176), ("f32", 300, 1152, 50021),
                                                       ("bf16", 700, 1152, 9001), ("bf16", 1500, 512, 100003)])
def test_confident_tokens(rows, width, vocab, dtype):
    """1 - p of about 1e-4 where the logits are about 300: both calls have the same logits, to the bit, so that what a sum of `width`
    products is off by does not count; only the rounding of lse does, and the sum of the exponentials."""
    gen = torch.Generator().manual_seed(14)
    w = torch.randn((vocab, width), generator=gen) * 2.5 * width ** -0.5
    w[:, 0] = 1.0
    w = w.to(TD[dtype])
    t = torch.randperm(vocab, generator=gen)[:rows]
    near = w[t].float()
    near[:, 0] = 0.0
    x = near * (math.log(vocab) + 9) / (near * near).sum(1, keepdim=True)
    x[:, 0] = 300.0
    i = dict(x=x.to(TD[dtype]).cuda(), w=w.cuda(), t=t.to(torch.int32).cuda(), g=torch.ones(rows, device="cuda"), ge=None)
    _, lse, _ = _forward(i, dtype)
    got = _backward(i, dtype, lse, None, ge=False)
    x, w, t = i["x"].double(), i["w"].double(), t.cuda()[:, None]
    logits, e = R.product(x, w)
    want_lse = torch.logsumexp(logits, 1, keepdim=True)
    p = (logits - want_lse).exp()
    rest = p.scatter(1, t, 0.0)  # (1 - p of the target, without a difference)
    missing = rest.sum(1, keepdim=True)
    d = (-rest).scatter(1, t, missing)
    # of the target: lse's rounding by half a step; the sum's roundings (as in ffn_ref.logprobs) and those of exponential and difference;
    # 1 - p itself by a logit's error at both ends.  Of others: p by the logit's and the lse's.
    off = 2.0 ** -24 * want_lse.abs() + R.U * (102 + vocab / 4096)
    e = e.amax(1, keepdim=True)
    ed = (rest * (2 * e + off)).scatter(1, t, off + missing * (2 * e + off))
    eps = R.half_step(TD[dtype])
    ed = ed + eps * (d.abs() + ed)
    for name, a, (c, ec) in zip(("d_hidden", "d_weight"), got, (R.product(d, w.T, ed), R.product(d.T, x.T, ed.T))):
        R.check(a, (c, ec + eps * (c.abs() + ec)), name)


@pytest.mark.parametrize("dtype, rows, width, vocab", [("bf16", 3, 8, (1 << 22) + 777), ("f32", 2, 16, (1 << 21) + 5)])
def test_vocabularies_of_millions(dtype, rows, width, vocab):
    """More tokens than a row of a piece's gradients has room for; targets on both sides of the pieces' borders."""
    i = _inputs(rows, width, vocab, dtype, seed=15)
    piece = ((vocab + 1) // 2 + 255) // 256 * 256
    i["t"] = torch.tensor([piece, piece - 1, vocab - 1][:rows], dtype=torch.int32, device="cuda")
    _check(i, dtype)
