"""Fine-tuning operators, host side (no GPU): tables of a batch of training sequences against the
fine-tuning mask's oracle, and what the calls refuse."""
import numpy as np
import pytest

from oracle import finetune_mask as FM
from paper_2604_26209_amd import binding as B

from finetune_ref import Batch


def _cfg(**kw):
    c = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, dtype=B.HPD_BF16, rope_base=10000.0, k_max=7,
             flags=B.HPD_FLAG_HOST_ONLY)
    c.update(kw)
    return B.hpd_finetune_config(*c.values())


def _build(batch, **kw):
    return B.hpd_build_finetune_layout(_cfg(k_max=batch.k_max, **kw), batch.prompt_len, batch.attr_ptr, batch.attr_len,
                                       batch.value_len)


def _status(call):
    with pytest.raises(B.HpdError) as e:
        call()
    return e.value.status


@pytest.mark.parametrize("seed", range(6))
def test_tables_equal_the_oracle(seed):
    batch = Batch.random(seed, 5, prompt=(0, 70), n_attr=(0, 9), k_max=3 + seed)
    lay = _build(batch)
    c = lay.counts()
    assert c[B.HPD_FTC_N_SEQ] == 5 and c[B.HPD_FTC_N_TOKENS] == batch.n and c[B.HPD_FTC_MAX_LEN] == max(batch.len)
    assert c[B.HPD_FTC_MAX_POS] == (batch.pos.max() if batch.n else -1)
    assert np.array_equal(B.hpd_finetune_layout_query(lay, B.HPD_FTQ_SEQ_OFF), batch.off)
    assert np.array_equal(B.hpd_finetune_layout_query(lay, B.HPD_FTQ_POS), batch.pos)
    rank = B.hpd_finetune_layout_query(lay, B.HPD_FTQ_RANK)
    for i, s in enumerate(batch.len):  # the mask as a comparison of ranks
        r, at = rank[batch.off[i]:batch.off[i + 1]], np.arange(s)
        seen = (at[None, :] <= at[:, None]) & (r[None, :] <= r[:, None])
        assert np.array_equal(seen, FM.finetune_mask(*batch.seqs[i]).astype(bool))


def test_empty_batches():
    for batch in (Batch([], 3), Batch([(0, [], [])], 3), Batch([(0, [], []), (0, [], [])], 3)):
        lay = _build(batch)
        assert lay.counts()[B.HPD_FTC_N_TOKENS] == 0 and lay.counts()[B.HPD_FTC_MAX_POS] == -1
        assert B.hpd_finetune_layout_query(lay, B.HPD_FTQ_POS).size == 0
        assert np.array_equal(B.hpd_finetune_layout_query(lay, B.HPD_FTQ_SEQ_OFF), batch.off)


@pytest.mark.parametrize("kw, status", [
    (dict(n_q_heads=0), B.HPD_E_INVALID), (dict(n_kv_heads=3), B.HPD_E_INVALID), (dict(head_dim=0), B.HPD_E_INVALID),
    (dict(head_dim=63), B.HPD_E_INVALID), (dict(k_max=0), B.HPD_E_INVALID), (dict(rope_base=1.0), B.HPD_E_INVALID),
    (dict(rope_base=float("nan")), B.HPD_E_INVALID), (dict(flags=2), B.HPD_E_INVALID),
    (dict(dtype=2), B.HPD_E_UNSUPPORTED), (dict(head_dim=60), B.HPD_E_UNSUPPORTED),
    (dict(head_dim=136), B.HPD_E_UNSUPPORTED)])
def test_refused_configurations(kw, status):
    assert _status(lambda: B.hpd_build_finetune_layout(_cfg(**kw), [3], [0, 1], [1], [1])) == status


def test_refused_batches():
    def build(*a, **kw):
        return _status(lambda: B.hpd_build_finetune_layout(_cfg(**kw), *a))
    assert build([-1], [0, 0], [], []) == B.HPD_E_INVALID
    assert build([1], [1, 1], [1], [1]) == B.HPD_E_INVALID       # attr_ptr[0]
    assert build([1, 1], [0, 2, 1], [1, 1], [1, 1]) == B.HPD_E_INVALID  # decreasing
    assert build([1], [0, 1], [0], [1]) == B.HPD_E_INVALID       # an empty name
    assert build([1], [0, 1], [1], [8]) == B.HPD_E_INVALID       # a value longer than k_max
    assert build([1], [0, 1], [1], [-1]) == B.HPD_E_INVALID
    assert build([2 ** 31 - 1], [0, 0], [], []) == B.HPD_E_OVERFLOW
    assert build([2 ** 25 + 1], [0, 0], [], [], n_q_heads=1, n_kv_heads=1) == B.HPD_E_OVERFLOW
    assert build([2 ** 24 + 1], [0, 0], [], []) == B.HPD_E_OVERFLOW  # times 8 heads
    assert build([1], [0, 2], [1, 1], [1, 1], k_max=2 ** 30) == B.HPD_E_OVERFLOW  # positions
    with pytest.raises(ValueError):
        B.hpd_build_finetune_layout(_cfg(), [1, 2], [0, 1], [1], [1])


def test_a_host_only_layout_runs_nothing():
    lay = _build(Batch([(4, [1], [2])], 3))
    x = 4096  # an address that nothing may touch
    assert _status(lambda: B.hpd_finetune_rotate(lay, 0, x, x, x, x, stream=0)) == B.HPD_E_INVALID
    assert _status(lambda: B.hpd_finetune_attention(lay, x, x, x, x, x, x, stream=0)) == B.HPD_E_INVALID
    assert _status(lambda: B.hpd_finetune_attention_backward(lay, x, x, x, x, x, x, x, x, x, x, stream=0)) == B.HPD_E_INVALID
    assert _status(lambda: B.hpd_finetune_layout_query(lay, 99)) == B.HPD_E_INVALID


def test_token_logprobs_refuses_bad_arguments():
    x = 4096

    def call(dtype=B.HPD_BF16, n=4, vocab=100, stride=100, logits=x, targets=x, top=0, lse=x, ids=x, tops=x, ws=x):
        return _status(lambda: B.hpd_token_logprobs(dtype, n, vocab, stride, logits, targets, top, x, lse, x, ids, tops, ws,
                                                    stream=0))
    assert call(dtype=7) == B.HPD_E_UNSUPPORTED
    assert call(n=-1) == B.HPD_E_INVALID
    assert call(vocab=0) == B.HPD_E_INVALID
    assert call(stride=99) == B.HPD_E_INVALID
    assert call(stride=2 ** 30 + 1) == B.HPD_E_OVERFLOW
    assert call(n=2 ** 30 + 1) == B.HPD_E_OVERFLOW
    assert call(logits=None) == B.HPD_E_INVALID
    assert call(logits=x + 1) == B.HPD_E_INVALID
    assert call(dtype=B.HPD_F32, logits=x + 2) == B.HPD_E_INVALID
    assert call(top=-1) == B.HPD_E_INVALID
    assert call(top=B.HPD_MAX_TOP + 1) == B.HPD_E_INVALID
    assert call(vocab=10, top=11) == B.HPD_E_INVALID
    assert call(top=3, ids=None) == B.HPD_E_INVALID
    assert call(top=3, tops=None) == B.HPD_E_INVALID
    assert call(vocab=10 ** 6, stride=10 ** 6, ws=None) == B.HPD_E_INVALID
    assert call(ws=x + 8) == B.HPD_E_INVALID
    B.hpd_token_logprobs(B.HPD_F32, 0, 10, 10, None, stream=0)  # no rows: nothing to do
    assert B.hpd_token_logprobs_workspace(B.HPD_F32, 0, 10 ** 6, 5) == 0
    assert B.hpd_token_logprobs_workspace(B.HPD_F32, 1, 10 ** 6, 5) > 0


def test_token_logprobs_backward_refuses_bad_arguments():
    x = 4096

    def call(dtype=B.HPD_BF16, n=4, vocab=100, stride=100, logits=x, targets=x, lse=x, ent=x, g=x, h=x, d=x, ds=100):
        return _status(lambda: B.hpd_token_logprobs_backward(dtype, n, vocab, stride, logits, targets, lse, ent, g, h, d, ds,
                                                             stream=0))
    assert call(dtype=7) == B.HPD_E_UNSUPPORTED
    assert call(n=-1) == B.HPD_E_INVALID
    assert call(vocab=-5) == B.HPD_E_INVALID
    assert call(stride=99) == B.HPD_E_INVALID
    assert call(ds=99) == B.HPD_E_INVALID
    assert call(logits=None) == B.HPD_E_INVALID
    assert call(d=None) == B.HPD_E_INVALID
    assert call(lse=None) == B.HPD_E_INVALID
    assert call(targets=None) == B.HPD_E_INVALID   # a gradient of log probabilities of no tokens
    assert call(ent=None) == B.HPD_E_INVALID       # the entropy's gradient needs the entropy
    assert call(d=x, stride=120, ds=100) == B.HPD_E_INVALID  # in place, but other rows
    assert call(d=x + 1) == B.HPD_E_INVALID
    B.hpd_token_logprobs_backward(B.HPD_F32, 0, 10, 10, None, None, None, None, None, None, None, 10, stream=0)
