"""Calls of fewer rows with the workspace of the most rows: nothing behind it is written, and the results are those with a workspace of
their own."""
import pytest
import torch

from paper_2604_26209_amd import binding as B
from test_gpu_ffn import DT, TD
from test_gpu_ffn import _inputs as _ffn_inputs
from test_gpu_head import _inputs as _head_inputs

pytestmark = pytest.mark.gpu

BEHIND = 4096


class Kept:
    """A workspace of `size` bytes with canaries behind it."""

    def __init__(self, size):
        self.buf = torch.full((size + BEHIND,), 0xa5, dtype=torch.uint8, device="cuda")
        self.t = self.buf[:size]
        self.t.fill_(0xff)  # (NaN in both types)

    def untouched(self):
        return bool((self.buf[-BEHIND:] == 0xa5).all())


def _equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


# the most rows, and fewer for which the contraction is cut into more parts than for those
@pytest.mark.parametrize("dtype, width, inner, most, fewer", [("bf16", 2048, 5504, 392, (391, 97, 1)), ("bf16", 1152, 2504, 2100, (2048, 513, 512)),
                                                              ("f32", 480, 1288, 700, (640, 33))])
def test_ffn(dtype, width, inner, most, fewer):
    cfg = B.hpd_ffn_config(width, inner, DT[dtype], B.HPD_ACT_SILU)
    kept = [Kept(n) for n in B.hpd_gated_ffn_workspace(cfg, most)]
    i = _ffn_inputs(most, width, inner, dtype, seed=21)

    def run(n, ws):
        outs = [torch.empty_like(i[k][:n]) for k in ("x", "g", "u", "x")] + [torch.empty_like(i[k]) for k in ("wg", "wu", "wd")]
        B.hpd_gated_ffn(cfg, n, i["x"], i["wg"], i["wu"], i["wd"], *outs[:3], ws[0])
        B.hpd_gated_ffn_backward(cfg, n, i["x"], i["wg"], i["wu"], i["wd"], outs[1], outs[2], i["d_out"], *outs[3:], ws[1])
        torch.cuda.synchronize()
        return outs

    for n in (most, *fewer):
        got = run(n, [k.t for k in kept])
        assert all(k.untouched() for k in kept), n
        assert _equal(got, run(n, [B.alloc_ffn_workspace(cfg, n, b) for b in (False, True)])), n


@pytest.mark.parametrize("dtype, width, vocab, most, fewer", [("bf16", 4096, 2057, 641, (640, 65, 1)), ("f32", 2048, 385, 900, (808, 130, 5)),
                                                              ("bf16", 256, 130013, 700, (513, 512, 2))])
def test_head(dtype, width, vocab, most, fewer):
    dt = DT[dtype]
    kept = [Kept(n) for n in B.hpd_head_logprobs_workspace(dt, most, width, vocab)]
    i = _head_inputs(most, width, vocab, dtype, seed=22)

    def run(n, ws):
        outs = [torch.empty(n, device="cuda") for _ in range(3)] + [torch.empty_like(i["x"][:n]), torch.empty_like(i["w"])]
        B.hpd_head_logprobs(dt, n, width, vocab, i["x"], 0, i["w"], 0, i["t"], *outs[:3], ws[0])
        B.hpd_head_logprobs_backward(dt, n, width, vocab, i["x"], 0, i["w"], 0, i["t"], outs[1], outs[2], i["g"], i["ge"], outs[3], 0,
                                     outs[4], 0, ws[1])
        torch.cuda.synchronize()
        return outs

    for n in (most, *fewer):
        got = run(n, [k.t for k in kept])
        assert all(k.untouched() for k in kept), n
        assert _equal(got, run(n, [B.alloc_head_workspace(dt, n, width, vocab, b) for b in (False, True)])), n
