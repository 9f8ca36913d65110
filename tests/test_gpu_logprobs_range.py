"""Token log probabilities over the whole range of finite logits, against the definition in 64 bits: tokens excluded by a finite
value of any size, rows of nothing else, rows whose largest logit is far from 0."""
import numpy as np
import pytest
import torch

import finetune_ref as R
from test_gpu_finetune import TD, _run_logprobs, _sum_error

pytestmark = pytest.mark.gpu

FILLS = [1e4, 2.0e6, 2.2e6, 3.0e6, 5e6, 1.7e7, 1e9, 1e10, 1e12, 1e20, 1e30, 5e37, 8e37, 9.5e37, 1e38, 3e38]


def _rows(fill, vocab, gen):
    """Rows of ordinary logits with a part at -fill or +fill."""
    at = torch.arange(vocab)
    part = min(8, vocab // 2)
    excluded = [at < part, at < vocab // 2, at >= vocab // 2, at >= vocab - max(1, vocab // 5), at % 3 == 1, at != vocab // 3,
                at >= 0]
    x = torch.randn((len(excluded) + 5, vocab), generator=gen) * 2.5
    for r, m in enumerate(excluded):
        x[r, m] = -fill
    a, b, c, d, e = range(len(excluded), len(excluded) + 5)
    x[a, vocab // 4] = fill                                # one logit above all
    x[b, :: max(1, vocab // 7)] = fill                     # some, equal
    x[c] += fill                                           # all of them, some steps apart
    x[d] -= fill
    x[e] = (x[e] * 1e4).clamp(-0.5, 0.5) * fill            # far apart on both sides of 0
    return x


def _compare(x, target, top):
    got = _run_logprobs(x.cuda(), torch.from_numpy(target.astype(np.int32)).cuda(), top)
    x64 = R.to_numpy(x)
    w_logprob, w_lse, w_ent, w_ids, w_vals = R.logprobs(x64, target, top)
    # the sum's terms and their reference point; a log probability has three more roundings, of numbers of its size
    error = _sum_error(x64, w_lse)
    R.check(got[1], w_lse, error + 2 * R.U32 * np.abs(w_lse), "lse")
    # (64 bits of lse: a step of it is not small against a difference of far logits)
    top_x = x64.max(1)
    log_sum = np.log(np.exp(x64 - top_x[:, None]).sum(1))
    has = (target >= 0) & (target < x.shape[1])
    w_logprob = np.where(has, x64[np.arange(len(x64)), np.where(has, target, 0)] - top_x - log_sum, 0.0)
    R.check(got[0], w_logprob, error + 4 * R.U32 * np.abs(w_logprob), "log probability")
    p = np.exp(x64 - top_x[:, None] - log_sum[:, None])
    apart = np.where(p > 0, x64 - top_x[:, None], 0.0)
    w_ent = log_sum - (p * apart).sum(1)
    R.check(got[2], w_ent, 3 * error * (1 + (p * np.abs(apart)).sum(1)), "entropy")
    assert np.array_equal(got[3].cpu().numpy(), w_ids)
    w_vals = np.take_along_axis(x64, w_ids.astype(np.int64), 1) - top_x[:, None] - log_sum[:, None]
    R.check(got[4], w_vals, error[:, None] + 4 * R.U32 * np.abs(w_vals), "alternatives")


# one wave per row, one workgroup per row, several pieces per row
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab, few", [(900, False), (4000, False), (8000, True), (32000, False), (128256, True)])
def test_finite_logits_of_any_size(vocab, few, dtype):
    gen = torch.Generator().manual_seed(vocab)
    for fill in FILLS[6::3] if few else FILLS:
        x = _rows(fill, vocab, gen).to(TD[dtype])
        target = np.arange(len(x)) * 977 % vocab
        target[1], target[7], target[9] = 0, vocab // 4, -1  # an excluded token, the largest, none
        _compare(x, target, 5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab", [(1, 33000), (1030, 9000)])
def test_rows_of_magnitudes_drawn_at_random(rows, vocab, dtype):
    """Signs and magnitudes from 1e-3 to 1e38 in every row, one piece or several."""
    rng = np.random.default_rng(rows)
    top = 10.0 ** rng.uniform(0, 38, (rows, 1))
    x = rng.choice([-1.0, 1.0], (rows, vocab)) * 10.0 ** rng.uniform(-3, np.log10(top), (rows, vocab))
    x[::2] = -np.abs(x[::2])                                # (the largest: near 0)
    x[1::4] = -top[1::4] + np.abs(x[1::4]) / 3              # (all far below 0)
    _compare(torch.from_numpy(x).to(TD[dtype]), rng.integers(0, vocab, rows), 4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1, 7, 64])
@pytest.mark.parametrize("vocab", [70, 900, 4000, 8000, 32000, 32768, 128256])
def test_alternatives_among_nan(vocab, top, dtype):
    """NaN counts as -infinity among the alternatives: the lowest indices come first where too few others are left."""
    inf = float("inf")
    x = torch.full((9, vocab), float("nan"))
    x[1, vocab - 1] = 2.0
    x[2, : min(5, top)] = torch.arange(min(5, top)) * 1.0
    x[3, vocab // 2:] = 0.5                        # enough others
    x[4, ::1000] = -torch.arange(len(x[4, ::1000])) * 1.0
    x[5, vocab // 3] = -inf                        # equal to the NaN around it
    x[6, vocab // 3] = -1.0e30
    x[7, vocab - 1] = inf
    x[8] = torch.randn(vocab, generator=torch.Generator().manual_seed(vocab))
    x[8, 8: vocab - vocab // 4] = float("nan")
    x = x.to(TD[dtype])
    target = torch.zeros(len(x), dtype=torch.int32, device="cuda")
    logprob, lse, entropy, ids, vals = _run_logprobs(x.cuda(), target, top)
    x64 = R.to_numpy(x)
    want = np.argsort(-np.where(np.isnan(x64), -np.inf, x64), axis=1, kind="stable")[:, :top]
    assert np.array_equal(ids.cpu().numpy(), want)
    for t in (logprob, lse, entropy, vals):
        assert bool(torch.isnan(t).all())
