"""The feed-forward block's and the vocabulary head's calls refuse what they cannot do before anything is enqueued."""
import ctypes

import pytest

from paper_2604_26209_amd import binding as B

P = [(k + 1) << 20 for k in range(16)]  # addresses that nothing reads


def _cfg(width=64, inner=40, dtype=B.HPD_BF16, act=B.HPD_ACT_SILU):
    return B.hpd_ffn_config(width, inner, dtype, act)


def _status(call, *args, **kw):
    with pytest.raises(B.HpdError) as e:
        call(*args, **kw, stream=0)
    return e.value.status


def _ffn(cfg=None, rows=5, x=P[0], wg=P[1], wu=P[2], wd=P[3], out=P[4], gate=P[5], up=P[6], ws=P[7], st=None):
    return _status(B.hpd_gated_ffn, cfg or _cfg(), rows, x, wg, wu, wd, out, gate, up, ws, st)


def _ffn_grad(cfg=None, rows=5, x=P[0], wg=P[1], wu=P[2], wd=P[3], gate=P[4], up=P[5], d_out=P[6], d_x=P[7], dwg=P[8], dwu=P[9],
              dwd=P[10], ws=P[11], st=None):
    return _status(B.hpd_gated_ffn_backward, cfg or _cfg(), rows, x, wg, wu, wd, gate, up, d_out, d_x, dwg, dwu, dwd, ws, st)


def _head(dtype=B.HPD_BF16, rows=5, width=64, vocab=33, x=P[0], sx=64, w=P[1], sw=64, t=P[2], lp=P[3], lse=P[4], ent=P[5], ws=P[6]):
    return _status(B.hpd_head_logprobs, dtype, rows, width, vocab, x, sx, w, sw, t, lp, lse, ent, ws)


def _head_grad(dtype=B.HPD_BF16, rows=5, width=64, vocab=33, x=P[0], sx=64, w=P[1], sw=64, t=P[2], lse=P[3], ent=P[4], g=P[5],
               ge=P[6], dx=P[7], sdx=64, dw=P[8], sdw=64, ws=P[9]):
    return _status(B.hpd_head_logprobs_backward, dtype, rows, width, vocab, x, sx, w, sw, t, lse, ent, g, ge, dx, sdx, dw, sdw, ws)


@pytest.mark.parametrize("call", [_ffn, _ffn_grad])
def test_ffn_configurations(call):
    assert call(_cfg(width=0)) == B.HPD_E_INVALID
    assert call(_cfg(inner=-8)) == B.HPD_E_INVALID
    assert call(_cfg(width=60)) == B.HPD_E_UNSUPPORTED
    assert call(_cfg(inner=44)) == B.HPD_E_UNSUPPORTED
    assert call(_cfg(dtype=2)) == B.HPD_E_UNSUPPORTED
    assert call(_cfg(act=3)) == B.HPD_E_UNSUPPORTED
    assert call(_cfg(act=-1)) == B.HPD_E_UNSUPPORTED
    assert call(_cfg(inner=1 << 22)) == B.HPD_E_OVERFLOW
    assert call(rows=-1) == B.HPD_E_INVALID
    assert call(rows=1 << 31) == B.HPD_E_OVERFLOW
    assert call(_cfg(inner=1 << 20), rows=1 << 20) == B.HPD_E_OVERFLOW


@pytest.mark.parametrize("name", ["x", "wg", "wu", "wd", "out", "ws"])
@pytest.mark.parametrize("value", [None, P[15] + 8])
def test_ffn_pointers(name, value):
    assert _ffn(**{name: value}) == B.HPD_E_INVALID


@pytest.mark.parametrize("name", ["x", "wg", "wu", "wd", "gate", "up", "d_out", "ws"])
@pytest.mark.parametrize("value", [None, P[15] + 8])
def test_ffn_grad_pointers(name, value):
    assert _ffn_grad(**{name: value}) == B.HPD_E_INVALID


def test_ffn_optional_pointers_and_overlaps():
    for name in ("gate", "up"):
        assert _ffn(**{name: P[15] + 4}) == B.HPD_E_INVALID
    for name in ("d_x", "dwg", "dwu", "dwd"):
        assert _ffn_grad(**{name: P[15] + 4}) == B.HPD_E_INVALID
    assert _ffn(out=P[0]) == B.HPD_E_INVALID
    assert _ffn(gate=P[5], up=P[5]) == B.HPD_E_INVALID
    assert _ffn(ws=P[4]) == B.HPD_E_INVALID
    assert _ffn_grad(d_x=P[6]) == B.HPD_E_INVALID
    assert _ffn_grad(dwg=P[1]) == B.HPD_E_INVALID
    assert _ffn_grad(dwd=P[11]) == B.HPD_E_INVALID


@pytest.mark.parametrize("name", [f for f, _ in B.hpd_ffn_strides._fields_])
def test_ffn_strides(name):
    for call in (_ffn, _ffn_grad):
        assert call(st=B.hpd_ffn_strides(**{name: 32})) == B.HPD_E_INVALID
        assert call(st=B.hpd_ffn_strides(**{name: 68})) == B.HPD_E_INVALID
        assert call(st=B.hpd_ffn_strides(**{name: -64})) == B.HPD_E_INVALID
        assert call(st=B.hpd_ffn_strides(**{name: 1 << 24})) == B.HPD_E_OVERFLOW


@pytest.mark.parametrize("call", [_head, _head_grad])
def test_head_sizes(call):
    assert call(dtype=7) == B.HPD_E_UNSUPPORTED
    assert call(width=0) == B.HPD_E_INVALID
    assert call(width=68, sx=72, sw=72) == B.HPD_E_UNSUPPORTED
    assert call(vocab=0) == B.HPD_E_INVALID
    assert call(rows=-1) == B.HPD_E_INVALID
    assert call(rows=1 << 31) == B.HPD_E_OVERFLOW
    assert call(rows=1 << 20, vocab=1 << 20) == B.HPD_E_OVERFLOW
    assert call(sx=32) == B.HPD_E_INVALID
    assert call(sw=66) == B.HPD_E_INVALID
    assert call(sw=1 << 23) == B.HPD_E_OVERFLOW


def test_head_pointers():
    for name in ("x", "w", "ws"):
        for value in (None, P[15] + 8):
            assert _head(**{name: value}) == B.HPD_E_INVALID
            assert _head_grad(**{name: value}) == B.HPD_E_INVALID
    for name in ("t", "lp", "lse", "ent"):
        assert _head(**{name: P[15] + 2}) == B.HPD_E_INVALID
    for name in ("t", "lse", "ent", "g", "ge"):
        assert _head_grad(**{name: P[15] + 2}) == B.HPD_E_INVALID
    for name in ("t", "lse", "ent"):
        assert _head_grad(**{name: None}) == B.HPD_E_INVALID
    for name in ("dx", "dw"):
        assert _head_grad(**{name: P[15] + 4}) == B.HPD_E_INVALID
    assert _head_grad(sdx=60) == B.HPD_E_INVALID
    assert _head_grad(sdw=60) == B.HPD_E_INVALID
    assert _head_grad(dx=P[0]) == B.HPD_E_INVALID
    assert _head_grad(dw=P[9]) == B.HPD_E_INVALID
    assert _head(lse=P[5], ent=P[5]) == B.HPD_E_INVALID


def test_calls_with_nothing_to_do():
    B.hpd_gated_ffn(_cfg(), 0, *[None] * 8, stream=0)
    B.hpd_gated_ffn_backward(_cfg(), 0, *[None] * 7, stream=0)
    B.hpd_gated_ffn_backward(_cfg(), 5, *P[:7], workspace=P[7], stream=0)
    B.hpd_head_logprobs(B.HPD_BF16, 0, 64, 33, None, 0, None, 0, stream=0)
    B.hpd_head_logprobs(B.HPD_BF16, 5, 64, 33, P[0], 0, P[1], 0, targets=None, logprob=P[2], workspace=P[3], stream=0)
    B.hpd_head_logprobs_backward(B.HPD_BF16, 5, 64, 33, P[0], 0, P[1], 0, P[2], P[3], None, P[4], None, workspace=P[5], stream=0)


def test_workspaces():
    assert B.hpd_gated_ffn_workspace(_cfg(), 0) == (0, 0)
    f, b = B.hpd_gated_ffn_workspace(_cfg(), 7)
    assert f >= 7 * 40 * 2 and b >= 3 * 7 * 40 * 2
    f32 = B.hpd_gated_ffn_workspace(_cfg(dtype=B.HPD_F32), 7)
    assert f32[0] >= 2 * 7 * 40 * 2 and f32[1] >= 6 * 7 * 40 * 2
    assert B.hpd_head_logprobs_workspace(B.HPD_BF16, 0, 64, 33) == (0, 0)
    # the logits of a large batch are never there as a whole
    rows, vocab = 6144, 130013
    f, b = B.hpd_head_logprobs_workspace(B.HPD_BF16, rows, 4096, vocab)
    assert 0 < f < rows * vocab * 2 / 10 and 0 < b < rows * vocab * 2 / 2
    for call, args in ((B._lib.hpd_gated_ffn_workspace, (ctypes.byref(_cfg(width=4)), 1)),
                       (B._lib.hpd_head_logprobs_workspace, (B.HPD_BF16, 1, 4, 9))):
        assert call(*args, None, None) == B.HPD_E_UNSUPPORTED
