"""The products of the feed-forward block and of the vocabulary head at sizes that take every shape of tile and every kind of cut: bounds by
likelihood, which an end or a stage that is lost or counted twice breaks (test_ffn_ref.py), and inputs of nothing but their ends."""
import pytest
import torch

import ffn_ref as R
from product_sizes import FFN, HEAD
from test_gpu_ffn import TD, _backward, _d, _forward, _inputs
from test_gpu_head import _backward as _head_backward
from test_gpu_head import _forward as _head_forward
from test_gpu_head import _inputs as _head_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, rows, width, inner", FFN)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_block(act, dtype, rows, width, inner):
    i = _inputs(rows, width, inner, dtype, seed=31)
    want = R.likely_ffn(*_d(i, "x", "wg", "wu", "wd"), act, TD[dtype])
    for name, a, w in zip(("out", "gate", "up"), _forward(i, rows, width, inner, dtype, act), want):
        R.check(a, w, name)
    del want
    want = R.likely_ffn_grad(*_d(i, "x", "wg", "wu", "wd", "g", "u", "d_out"), act, TD[dtype])
    for name, a, w in zip(("dx", "dw_gate", "dw_up", "dw_down"), _backward(i, rows, width, inner, dtype, act), want):
        R.check(a, w, name)


@pytest.mark.parametrize("dtype, rows, width, inner", FFN)
def test_block_of_nothing_but_ends(dtype, rows, width, inner):
    """The last eight of every contracted index, or the last row, are all that is there."""
    i = _inputs(rows, width, inner, dtype, seed=32)
    i["x"][:, :-8] = 0
    i["wd"][:, :-8] = 0
    want = R.ffn(*_d(i, "x", "wg", "wu", "wd"), "silu", TD[dtype])
    for name, a, w in zip(("out", "gate", "up"), _forward(i, rows, width, inner, dtype, "silu"), want):
        R.check(a, w, name)
    i["d_out"][:, :-8] = 0
    for all_rows in (True, False):
        if not all_rows:
            i["x"], i["d_out"] = _inputs(rows, width, inner, dtype, seed=33)["x"], i["d_out"].clone()
            i["d_out"][:-1] = 0
        want = R.ffn_grad(*_d(i, "x", "wg", "wu", "wd", "g", "u", "d_out"), "silu", TD[dtype])
        for name, a, w in zip(("dx", "dw_gate", "dw_up", "dw_down"), _backward(i, rows, width, inner, dtype, "silu"), want):
            R.check(a, w, name)


@pytest.mark.parametrize("dtype, rows, width, vocab", HEAD)
def test_head(dtype, rows, width, vocab):
    """Targets among the last tokens."""
    i = _head_inputs(rows, width, vocab, dtype, seed=34)
    i["t"] = (vocab - 1 - torch.arange(rows, device="cuda") % min(64, vocab)).int()
    x, w = i["x"].double(), i["w"].double()
    got = _head_forward(i, dtype)
    for name, a, want in zip(("logprob", "lse", "entropy"), got, R.likely_head(x, w, i["t"])):
        R.check(a, want, name)
    want = R.likely_head_grad(x, w, i["t"], i["g"].double(), TD[dtype])
    for name, a, b in zip(("d_hidden", "d_weight"), _head_backward(i, dtype, got[1], None, ge=False), want):
        R.check(a, b, name)


@pytest.mark.parametrize("dtype, rows, width, vocab", HEAD)
def test_head_of_nothing_but_ends(dtype, rows, width, vocab):
    """The last eight channels of the hidden states; the last token's weights are all that its row's gradient comes from."""
    i = _head_inputs(rows, width, vocab, dtype, seed=35)
    i["x"][:, :-8] = 0
    i["t"] = torch.full((rows,), vocab - 1, dtype=torch.int32, device="cuda")
    x, w = i["x"].double(), i["w"].double()
    got = _head_forward(i, dtype)
    for name, a, want in zip(("logprob", "lse", "entropy"), got, R.likely_head(x, w, i["t"])):
        R.check(a, want, name)
    i["g"][:-1] = 0
    want = R.head_grad(x, w, i["t"], got[1].double(), None, i["g"].double(), None, TD[dtype])
    for name, a, b in zip(("d_hidden", "d_weight"), _head_backward(i, dtype, got[1], None, ge=False), want):
        R.check(a, b, name)
