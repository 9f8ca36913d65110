"""The gated feed-forward block and its gradient through the library, against the formulas in 64 bits."""
import pytest
import torch

import ffn_ref as R
from paper_2604_26209_amd import binding as B

pytestmark = pytest.mark.gpu

TD = dict(f32=torch.float32, bf16=torch.bfloat16)
DT = dict(f32=B.HPD_F32, bf16=B.HPD_BF16)
ACTS = dict(silu=B.HPD_ACT_SILU, gelu=B.HPD_ACT_GELU, gelu_tanh=B.HPD_ACT_GELU_TANH)
GUARD = 8  # elements of canary around every row


class Padded:
    """A matrix inside a buffer of canaries: rows further apart than they are long, something before and behind."""

    def __init__(self, rows, cols, dtype, fill=None, pad=GUARD):
        self.rows, self.cols, self.pad = rows, cols, pad
        self.buf = torch.full((rows + 2, cols + 2 * pad), 31744.0, dtype=dtype, device="cuda")
        self.t = self.buf[1:rows + 1, pad:pad + cols] if pad else self.buf[1:rows + 1]
        if fill is not None:
            self.t.copy_(fill)

    def untouched(self):
        inner = torch.zeros_like(self.buf, dtype=torch.bool)
        inner[1:self.rows + 1, self.pad:self.pad + self.cols] = True
        return bool((self.buf[~inner] == 31744.0).all())


def _inputs(rows, width, inner, dtype, seed=0, scale=1.0):
    gen = torch.Generator().manual_seed(seed)

    def normal(r, c, std):
        return (torch.randn((r, c), generator=gen) * std).to(TD[dtype]).cuda()

    return dict(x=normal(rows, width, scale), wg=normal(inner, width, width ** -0.5), wu=normal(inner, width, width ** -0.5),
                wd=normal(width, inner, inner ** -0.5), g=normal(rows, inner, 1.5), u=normal(rows, inner, 1.0),
                d_out=normal(rows, width, 0.1))


def _forward(i, rows, width, inner, dtype, act, keep=True, pad=GUARD):
    cfg = B.hpd_ffn_config(width, inner, DT[dtype], ACTS[act])
    t = {k: Padded(*i[k].shape, TD[dtype], i[k], pad) for k in ("x", "wg", "wu", "wd")}
    out = Padded(rows, width, TD[dtype], pad=pad)
    gate, up = (Padded(rows, inner, TD[dtype], pad=pad) for _ in range(2))
    ws = B.alloc_ffn_workspace(cfg, rows, backward=False)
    st = B.hpd_ffn_strides(x=t["x"].t.stride(0), out=out.t.stride(0), gate=gate.t.stride(0), up=up.t.stride(0),
                           w_gate=t["wg"].t.stride(0), w_up=t["wu"].t.stride(0), w_down=t["wd"].t.stride(0))
    B.hpd_gated_ffn(cfg, rows, t["x"].t, t["wg"].t, t["wu"].t, t["wd"].t, out.t, gate.t if keep else None,
                    up.t if keep else None, ws, st)
    torch.cuda.synchronize()
    assert all(p.untouched() for p in (out, gate, up))
    return out.t, gate.t, up.t


def _backward(i, rows, width, inner, dtype, act, wanted=(True,) * 4, pad=GUARD):
    cfg = B.hpd_ffn_config(width, inner, DT[dtype], ACTS[act])
    t = {k: Padded(*i[k].shape, TD[dtype], i[k], pad) for k in ("x", "wg", "wu", "wd", "g", "u", "d_out")}
    dx, dwg, dwu, dwd = (Padded(r, c, TD[dtype], pad=pad) for r, c in ((rows, width), (inner, width), (inner, width), (width, inner)))
    ws = B.alloc_ffn_workspace(cfg, rows, backward=True)
    if ws is not None:
        ws.fill_(0xff)  # (NaN in both types)
    st = B.hpd_ffn_strides(**{a: t[b].t.stride(0) for a, b in (("x", "x"), ("w_gate", "wg"), ("w_up", "wu"), ("w_down", "wd"),
                                                               ("gate", "g"), ("up", "u"), ("d_out", "d_out"))},
                           d_x=dx.t.stride(0), d_w_gate=dwg.t.stride(0), d_w_up=dwu.t.stride(0), d_w_down=dwd.t.stride(0))
    outs = (dx, dwg, dwu, dwd)
    B.hpd_gated_ffn_backward(cfg, rows, t["x"].t, t["wg"].t, t["wu"].t, t["wd"].t, t["g"].t, t["u"].t, t["d_out"].t,
                             *[o.t if w else None for o, w in zip(outs, wanted)], ws, st)
    torch.cuda.synchronize()
    for o, w in zip(outs, wanted):
        assert o.untouched()
        assert w or bool((o.buf == 31744.0).all())
    return [o.t for o in outs]


def _d(i, *names):
    return [i[n].double() for n in names]


SIZES = [(1, 8, 8), (2, 64, 40), (31, 72, 264), (33, 136, 128), (64, 256, 200), (65, 64, 8), (100, 1000, 328), (129, 480, 1288),
         (257, 512, 520), (300, 128, 1032)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, width, inner", SIZES)
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_forward(rows, width, inner, act, dtype):
    i = _inputs(rows, width, inner, dtype)
    want = R.ffn(*_d(i, "x", "wg", "wu", "wd"), act, TD[dtype])
    for name, got, w in zip(("out", "gate", "up"), _forward(i, rows, width, inner, dtype, act), want):
        R.check(got, w, name)
    out, gate, up = _forward(i, rows, width, inner, dtype, act, keep=False, pad=0)
    R.check(out, want[0], "out")
    assert bool((gate == 31744.0).all() and (up == 31744.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, width, inner", SIZES)
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_backward(rows, width, inner, act, dtype):
    i = _inputs(rows, width, inner, dtype, seed=1)
    want = R.ffn_grad(*_d(i, "x", "wg", "wu", "wd", "g", "u", "d_out"), act, TD[dtype])
    for name, got, w in zip(("dx", "dw_gate", "dw_up", "dw_down"), _backward(i, rows, width, inner, dtype, act), want):
        R.check(got, w, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("wanted", [(1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (1, 1, 0, 1), (0, 0, 1, 1)])
def test_gradients_that_are_not_wanted(wanted, dtype):
    rows, width, inner = 70, 136, 264
    i = _inputs(rows, width, inner, dtype, seed=2)
    want = R.ffn_grad(*_d(i, "x", "wg", "wu", "wd", "g", "u", "d_out"), "silu", TD[dtype])
    for got, w, on in zip(_backward(i, rows, width, inner, dtype, "silu", wanted), want, wanted):
        if on:
            R.check(got, w, str(wanted))


# many rows, as in a training batch; the whole chain from forward to backward in larger sizes
@pytest.mark.parametrize("dtype, rows, width, inner", [("bf16", 2049, 1152, 2504), ("bf16", 512, 4096, 2056), ("bf16", 3, 4096, 8200),
                                                       ("f32", 1025, 480, 1288), ("bf16", 5000, 256, 520), ("bf16", 96, 2048, 5504)])
def test_larger(dtype, rows, width, inner):
    i = _inputs(rows, width, inner, dtype, seed=3)
    want = R.ffn(*_d(i, "x", "wg", "wu", "wd"), "silu", TD[dtype])
    got = _forward(i, rows, width, inner, dtype, "silu", pad=0)
    for name, a, w in zip(("out", "gate", "up"), got, want):
        R.check(a, w, name)
    i["g"], i["u"] = got[1].clone(), got[2].clone()
    want = R.ffn_grad(*_d(i, "x", "wg", "wu", "wd", "g", "u", "d_out"), "silu", TD[dtype])
    for name, a, w in zip(("dx", "dw_gate", "dw_up", "dw_down"), _backward(i, rows, width, inner, dtype, "silu"), want):
        R.check(a, w, name)


# tiles of every size in every product, whole and cut contractions, ends of all kinds
@pytest.mark.parametrize("dtype, rows, width, inner", [("bf16", 4100, 2048, 4104), ("bf16", 2049, 4096, 4104), ("bf16", 700, 4096, 8200),
                                                       ("bf16", 8200, 1032, 2504), ("bf16", 32, 4096, 8200), ("f32", 3, 4096, 8200),
                                                       ("f32", 32, 1152, 4008), ("f32", 64, 2048, 2056), ("bf16", 64, 1160, 12296)])
def test_tiles_of_every_size(dtype, rows, width, inner):
    i = _inputs(rows, width, inner, dtype, seed=8)
    want = R.ffn(*_d(i, "x", "wg", "wu", "wd"), "gelu_tanh", TD[dtype])
    for name, a, w in zip(("out", "gate", "up"), _forward(i, rows, width, inner, dtype, "gelu_tanh"), want):
        R.check(a, w, name)
    del want
    want = R.ffn_grad(*_d(i, "x", "wg", "wu", "wd", "g", "u", "d_out"), "gelu_tanh", TD[dtype])
    for name, a, w in zip(("dx", "dw_gate", "dw_up", "dw_down"), _backward(i, rows, width, inner, dtype, "gelu_tanh"), want):
        R.check(a, w, name)


# 64 x 128 tiles in each product, 192 x 256 with odd ends, a middle number of rows
@pytest.mark.parametrize("dtype, rows, width, inner", [("bf16", 100, 4096, 6008), ("bf16", 120, 2048, 8200), ("bf16", 65, 4104, 4104),
                                                       ("bf16", 1001, 2048, 8200), ("bf16", 509, 4096, 12296)])
def test_tiles_between(dtype, rows, width, inner):
    test_tiles_of_every_size(dtype, rows, width, inner)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 130])
def test_halves_of_one_matrix(rows, dtype):
    """Both projections in one matrix, what is kept in one buffer, their gradients in one: the same bits."""
    width, inner, td = 136, 264, TD[dtype]
    i = _inputs(rows, width, inner, dtype, seed=9)
    cfg = B.hpd_ffn_config(width, inner, DT[dtype], ACTS["silu"])
    w = torch.cat([i["wg"], i["wu"]])
    kept, d_w = torch.empty((rows, 2 * inner), dtype=td, device="cuda"), torch.empty_like(w)
    out, dx, dwd = torch.empty_like(i["x"]), torch.empty_like(i["x"]), torch.empty_like(i["wd"])
    st = B.hpd_ffn_strides(gate=2 * inner, up=2 * inner)
    ws = [B.alloc_ffn_workspace(cfg, rows, b) for b in (False, True)]
    g, u = kept[:, :inner], kept[:, inner:]
    B.hpd_gated_ffn(cfg, rows, i["x"], w[:inner], w[inner:], i["wd"], out, g, u, ws[0], st)
    a, b, c = _forward(i, rows, width, inner, dtype, "silu")
    assert torch.equal(out, a) and torch.equal(g, b) and torch.equal(u, c)
    B.hpd_gated_ffn_backward(cfg, rows, i["x"], w[:inner], w[inner:], i["wd"], g, u, i["d_out"], dx, d_w[:inner], d_w[inner:], dwd,
                             ws[1], st)
    i["g"], i["u"] = b, c
    for x, y in zip((dx, d_w[:inner], d_w[inner:], dwd), _backward(i, rows, width, inner, dtype, "silu")):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype, rows, width, inner", [("bf16", 509, 4096, 12288), ("bf16", 515, 256, 520), ("f32", 300, 264, 136)])
def test_rows_8_mb_apart(dtype, rows, width, inner):
    """The widest strides, more than 4 GB from the first row to the last in bf16: the bits of rows without gaps."""
    i, cfg = _inputs(rows, width, inner, dtype, seed=12), B.hpd_ffn_config(width, inner, DT[dtype], ACTS["silu"])
    stride = (8 << 20) // i["x"].element_size()
    far = torch.empty((rows, stride), dtype=TD[dtype], device="cuda")
    x, out, d_out, dx = (far[:, k * width:(k + 1) * width] for k in range(4))
    gate, up = (far[:, k:k + inner] for k in (stride // 2, stride // 2 + inner))
    x.copy_(i["x"])
    d_out.copy_(i["d_out"])
    st = B.hpd_ffn_strides(x=stride, out=stride, gate=stride, up=stride, d_out=stride, d_x=stride)
    ws = [B.alloc_ffn_workspace(cfg, rows, b) for b in (False, True)]
    grads = [torch.empty_like(i[k]) for k in ("wg", "wu", "wd")]
    B.hpd_gated_ffn(cfg, rows, x, i["wg"], i["wu"], i["wd"], out, gate, up, ws[0], st)
    B.hpd_gated_ffn_backward(cfg, rows, x, i["wg"], i["wu"], i["wd"], gate, up, d_out, dx, *grads, ws[1], st)
    near = [torch.empty_like(i[k]) for k in ("x", "g", "u", "x", "wg", "wu", "wd")]
    B.hpd_gated_ffn(cfg, rows, i["x"], i["wg"], i["wu"], i["wd"], *near[:3], ws[0])
    B.hpd_gated_ffn_backward(cfg, rows, i["x"], i["wg"], i["wu"], i["wd"], near[1], near[2], i["d_out"], *near[3:], ws[1])
    for a, b in zip((out, gate, up, dx, *grads), near):
        assert torch.equal(a, b)


def test_two_calls_at_once():
    """Calls on two streams with workspaces of their own."""
    rows, width, inner = 257, 512, 1032
    inputs = [_inputs(rows, width, inner, "bf16", seed=s) for s in (10, 11)]
    want = [[t.clone() for t in _forward(i, rows, width, inner, "bf16", "silu", pad=0)] for i in inputs]
    cfg = B.hpd_ffn_config(width, inner, B.HPD_BF16, B.HPD_ACT_SILU)
    ws = [B.alloc_ffn_workspace(cfg, rows, False) for _ in inputs]
    outs = [[torch.empty_like(t) for t in w] for w in want]
    streams = [torch.cuda.Stream() for _ in inputs]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, w, o, s in zip(inputs, ws, outs, streams):
            B.hpd_gated_ffn(cfg, rows, i["x"], i["wg"], i["wu"], i["wd"], *o, w, stream=s)
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_no_rows():
    """Nothing to do but the weights' gradients: zeros."""
    i = _inputs(0, 64, 40, "bf16")
    _forward(i, 0, 64, 40, "bf16", "silu")
    _, *grads = _backward(i, 0, 64, 40, "bf16", "silu")
    assert all(bool((g == 0).all()) for g in grads)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 150])
def test_a_row_that_is_not_finite_stays_alone(rows, dtype):
    width, inner = 136, 264
    i = _inputs(rows, width, inner, dtype, seed=4)
    clean = [t.clone() for t in _forward(i, rows, width, inner, dtype, "silu")]
    back = _backward(i, rows, width, inner, dtype, "silu", (1, 0, 0, 0))[0].clone()
    for bad in (float("nan"), float("inf")):
        j = dict(i, x=i["x"].clone(), d_out=i["d_out"].clone())
        j["x"][3, 5] = bad
        j["d_out"][3, 5] = bad
        keep = torch.arange(rows, device="cuda") != 3
        for a, b in zip(_forward(j, rows, width, inner, dtype, "silu"), clean):
            assert torch.equal(a[keep], b[keep]) and not bool(torch.isfinite(a[3]).all())
        a = _backward(j, rows, width, inner, dtype, "silu", (1, 0, 0, 0))[0]
        assert torch.equal(a[keep], back[keep]) and not bool(torch.isfinite(a[3]).all())


@pytest.mark.parametrize("act", list(ACTS))
def test_activations_far_out(act):
    """Large and tiny values of g through all activations, exactly where the result is 0 or g."""
    g = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e-4, -1e-4, 0.5, -0.5, 3.0, -3.0, 9.0, -9.0, 30.0, -30.0, 90.0, -90.0, 1e4,
                      -1e4, 1e10, -1e10, 1e12, -1e12, 2.0, -2.0])
    width = inner = 24
    eye = torch.eye(width)
    i = dict(x=torch.diag(g).cuda(), wg=eye.cuda(), wu=torch.ones((inner, width)).cuda() / g.abs().clamp(min=1e-20)[None].cuda(),
             wd=eye.cuda(), g=g[None].cuda().contiguous(), u=torch.ones((1, inner)).cuda(), d_out=torch.ones((1, width)).cuda())
    out, gate, up = _forward(i, width, width, inner, "f32", act)
    a, slope = R.act(g.double(), act)
    want = a * up.double().cpu().diagonal()
    got = out.double().cpu().diagonal()
    # (a gelu that is tiny next to g comes from a difference; a logistic function under the smallest normal number, 2^-126, is
    # 0: exp(-g) above 2^128 is infinity in fp32)
    bound = 1e-5 * want.abs() + (g * up.cpu().diagonal()).abs().double() * (2e-7 * (g.abs() < 30) + 2.0 ** -126)
    assert bool(((got - want).abs() <= bound).all()), (got, want)
    dx = _backward(i, 1, width, inner, "f32", act, (1, 0, 0, 0))[0].double().cpu()[0]
    du = a
    want = slope + (du[None] @ i["wu"].double().cpu())[0]
    # dx = dg + a's sum over the up projection
    bound = R.FUNC * (1 + g.double().abs() * (g.abs() < 30)) + 1e-5 * (du.abs()[None] @ i["wu"].double().cpu().abs())[0]
    assert bool(((dx - want).abs() <= bound).all()), (dx, want)


@pytest.mark.parametrize("rows", [3, 200])
def test_equal_calls_give_equal_bits_on_any_stream_and_in_a_graph(rows):
    width, inner, dtype = 264, 520, torch.bfloat16
    i = _inputs(rows, width, inner, "bf16", seed=5)
    cfg = B.hpd_ffn_config(width, inner, B.HPD_BF16, B.HPD_ACT_SILU)

    def empty(*s):
        return torch.full(s, float("nan"), dtype=dtype, device="cuda")

    out, g, u = empty(rows, width), empty(rows, inner), empty(rows, inner)
    grads = [empty(rows, width), empty(inner, width), empty(inner, width), empty(width, inner)]
    ws = [B.alloc_ffn_workspace(cfg, rows, b) for b in (False, True)]

    def step():
        B.hpd_gated_ffn(cfg, rows, i["x"], i["wg"], i["wu"], i["wd"], out, g, u, ws[0])
        B.hpd_gated_ffn_backward(cfg, rows, i["x"], i["wg"], i["wu"], i["wd"], g, u, i["d_out"], *grads, ws[1])

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (out, g, u, *grads)]

    def forget():
        for t in (out, g, u, *grads):
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
        if n % 2 == 0:
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_gradients_against_differences():
    """A directional derivative of a weighted sum of the outputs, fp32."""
    rows, width, inner, act = 17, 72, 136, "gelu"
    i = _inputs(rows, width, inner, "f32", seed=6)
    _, i["g"], i["u"] = (t.clone() for t in _forward(i, rows, width, inner, "f32", act))
    grads = _backward(i, rows, width, inner, "f32", act)
    gen = torch.Generator().manual_seed(7)
    for name, d in zip(("x", "wg", "wu", "wd"), grads):
        way = torch.randn(i[name].shape, generator=gen).cuda()
        sums = []
        for h in (-1, 1):
            j = {k: v.double() for k, v in i.items()}
            j[name] = j[name] + h * 1e-4 * way.double()
            a = R.act(j["x"] @ j["wg"].T, act)[0] * (j["x"] @ j["wu"].T)
            sums.append(((a @ j["wd"].T) * i["d_out"].double()).sum().item())
        numeric, analytic = (sums[1] - sums[0]) / 2e-4, (d.double() * way.double()).sum().item()
        # third derivatives of order 10 times 1e-8, and the gradient's own roundings over its elements
        assert abs(numeric - analytic) <= 1e-5 * (d.double() * way.double()).abs().sum().item() + 1e-5, name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", list(ACTS))
def test_activations_at_the_ends_of_the_range(act, dtype):
    """Any finite g: act(g) is g or 0 and its slope 1 or 0, though squares and multiples of g overflow; act(+infinity) is +infinity."""
    g = torch.tensor([1e12, 1e19, 2e19, 3e19, 1e25, 1e30, 1.2e38, 2e38, 2.4e38, 3e38, 3.3e38, 30.0])
    g = torch.cat([g, -g]).to(TD[dtype])
    n = len(g)
    eye, none = torch.eye(n), torch.zeros((n, n))
    i = dict(x=torch.cat([torch.diag(g.float()), eye / 16], 1), wg=torch.cat([eye, none], 1), wu=torch.cat([none, eye], 1),
             wd=torch.cat([eye, none]), g=g[None].float(), u=torch.ones((1, n)), d_out=torch.ones((1, 2 * n)))
    i = {k: v.to(TD[dtype]).cuda().contiguous() for k, v in i.items()}
    out, gate, up = _forward(i, n, 2 * n, n, dtype, act)
    assert torch.equal(gate.cpu(), torch.diag(g)) and bool((up.diagonal() == 1 / 16).all())
    want = torch.where(g > 0, g, 0.0).double() / 16
    got = out.double().cpu().diagonal()
    assert bool(((got - want).abs() <= R.FUNC * want + 1e-11).all()), (got, want)
    j = dict(i, wu=torch.zeros_like(i["wu"]))
    dx = _backward(j, 1, 2 * n, n, dtype, act, (1, 0, 0, 0))[0].double().cpu()[0, :n]
    assert bool(((dx - (g > 0).double()).abs() <= R.FUNC + R.half_step(TD[dtype])).all()), dx
    # a sum that overflows in the gate
    i = {k: torch.zeros((8, 8)) for k in ("x", "wg", "wu", "wd")}
    i["x"][0, 0], i["wg"][0, 0], i["wu"][0, 0] = 3e38, 2.0, 2.0 ** -126
    i["wd"] += 1.0
    out, gate, _ = _forward({k: v.to(TD[dtype]).cuda() for k, v in i.items()}, 8, 8, 8, dtype, act)
    assert float(gate[0, 0]) == float("inf") and bool((out[0] == float("inf")).all()) and bool((out[1:] == 0).all())
