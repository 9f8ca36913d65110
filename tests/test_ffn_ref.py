"""The bounds by likelihood of ffn_ref: arithmetic as the kernels do it stays within them, and what a lost end or stage of a contraction
leaves does not, at every size that the GPU tests of whole contractions run."""
import pytest
import torch

import ffn_ref as R
from product_sizes import FFN, HEAD

TD = dict(f32=torch.float32, bf16=torch.bfloat16)
STAGE = dict(f32=32, bf16=64)


def _normal(gen, dtype, r, c, std):
    return (torch.randn((r, c), generator=gen) * std).to(TD[dtype]).double()


def _off(got, want):
    value, bound = want
    return not bool(((got - value).abs() <= bound).all())


def _as(v, dtype):
    return v.to(TD[dtype]).double()


def _product32(a, b):
    return (a.float() @ b.float().T).double()


@pytest.mark.parametrize("dtype, rows, width, inner", FFN)
def test_block(dtype, rows, width, inner):
    """Each contraction at its full length, the other sizes cut down to 64."""
    gen = torch.Generator().manual_seed(1)
    few, stage = min(rows, 64), STAGE[dtype]
    for d, f in ((64, inner), (width, 64)):
        x = _normal(gen, dtype, few, d, 1.0)
        wg, wu = (_normal(gen, dtype, f, d, d ** -0.5) for _ in range(2))
        wd = _normal(gen, dtype, d, f, f ** -0.5)
        out, gate, up = R.likely_ffn(x, wg, wu, wd, "gelu_tanh", TD[dtype])
        g, u = _product32(x, wg), _product32(x, wu)
        h = _as(R.act(g, "gelu_tanh")[0] * u, dtype)
        assert not _off(_as(g, dtype), gate) and not _off(_as(u, dtype), up) and not _off(_as(_product32(h, wd), dtype), out)
        for lost in (slice(-8, None), slice(0, stage), slice(f // 2 // 8 * 8, f // 2 // 8 * 8 + stage)):
            if f == inner:
                a = h.clone()
                a[:, lost] = 0
                assert _off(_as(_product32(a, wd), dtype), out), lost
            else:
                a = x.clone()
                a[:, lost] = 0
                assert _off(_as(_product32(a, wg), dtype), gate), lost
        g, u, d_out = _normal(gen, dtype, few, f, 1.5), _normal(gen, dtype, few, f, 1.0), _normal(gen, dtype, few, d, 0.1)
        dx, _, _, _ = R.likely_ffn_grad(x, wg, wu, wd, g, u, d_out, "gelu_tanh", TD[dtype])
        a, slope = R.act(g, "gelu_tanh")

        def of_x(dh, lost=slice(0, 0)):
            dg, du = _as(dh * u * slope, dtype), _as(dh * a, dtype)
            both = torch.cat([dg, du], 1)
            both[:, lost] = 0
            return _as(_product32(both, torch.cat([wg, wu], 0).T), dtype)
        dh = _product32(d_out, wd.T)
        assert not _off(of_x(dh), dx)
        if f == inner:
            for lost in (slice(-8, None), slice(f - 8, f), slice(f, f + stage)):
                assert _off(of_x(dh, lost), dx), lost
        else:
            part = d_out.clone()
            part[:, -8:] = 0
            assert _off(of_x(_product32(part, wd.T)), dx)
    # the weights' gradients
    d = f = 64
    x, d_out = _normal(gen, dtype, rows, d, 1.0), _normal(gen, dtype, rows, d, 0.1)
    wg, wu, wd = _normal(gen, dtype, f, d, d ** -0.5), _normal(gen, dtype, f, d, d ** -0.5), _normal(gen, dtype, d, f, f ** -0.5)
    g, u = _normal(gen, dtype, rows, f, 1.5), _normal(gen, dtype, rows, f, 1.0)
    _, dwg, dwu, dwd = R.likely_ffn_grad(x, wg, wu, wd, g, u, d_out, "gelu_tanh", TD[dtype])
    a, slope = R.act(g, "gelu_tanh")
    dh = _product32(d_out, wd.T)
    h, dg, du = _as(a * u, dtype), _as(dh * u * slope, dtype), _as(dh * a, dtype)
    for p, q, want in ((dg.T, x.T, dwg), (du.T, x.T, dwu), (d_out.T, h.T, dwd)):
        assert not _off(_as(_product32(p, q), dtype), want)
        assert _off(_as(_product32(p[:, :-1], q[:, :-1]), dtype), want)


@pytest.mark.parametrize("dtype, rows, width, vocab", HEAD)
def test_head(dtype, rows, width, vocab):
    """Targets among the last tokens: their rows of the weights carry the gradients."""
    gen = torch.Generator().manual_seed(2)
    few = min(rows, 48)
    x, w = _normal(gen, dtype, few, width, 1.0), _normal(gen, dtype, 512, width, 2.5 * width ** -0.5)
    t = 511 - torch.arange(few) % 64
    logprob, lse, _ = R.likely_head(x, w, t)
    logits = _product32(x, w)
    got = torch.logsumexp(logits, 1)
    at = t[:, None]
    assert not _off(_as(got, "f32"), lse) and not _off((logits - got[:, None]).gather(1, at)[:, 0], logprob)
    part = _product32(x[:, :-8], w[:, :-8])
    assert _off((part - torch.logsumexp(part, 1, keepdim=True)).gather(1, at)[:, 0], logprob)
    g = torch.randn(few, generator=gen).double()
    dx, dw = R.likely_head_grad(x, w, t, g, TD[dtype])
    hot = torch.zeros_like(logits).scatter_(1, at, 1.0)
    d = _as(g[:, None] * (hot - (logits - got[:, None]).exp()), dtype)
    assert not _off(_as(_product32(d, w.T), dtype), dx) and not _off(_as(_product32(d.T, x.T), dtype), dw)
    assert _off(_as(_product32(d[:, :-1], w[:-1].T), dtype), dx)
    assert _off(_as(_product32(d[:-1].T, x[:-1].T), dtype), dw)
