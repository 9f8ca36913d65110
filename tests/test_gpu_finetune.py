"""Fine-tuning operators on the GPU against their definitions in 64 bits (tests/finetune_ref.py), element by
element within bounds that count the roundings."""
import numpy as np
import pytest
import torch

import finetune_ref as R
from finetune_ref import Batch

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "bf16": torch.bfloat16}


def _dtype(name):
    from paper_2604_26209_amd import binding as B
    return B.HPD_F32 if name == "f32" else B.HPD_BF16


def _layout(batch, hq, hkv, d, dtype, base=10000.0):
    from paper_2604_26209_amd import binding as B
    cfg = B.hpd_finetune_config(hq, hkv, d, _dtype(dtype), base, batch.k_max, 0)
    return B.hpd_build_finetune_layout(cfg, batch.prompt_len, batch.attr_ptr, batch.attr_len, batch.value_len)


def _normal(seed, shape, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(TD[dtype])


class Run:
    """q, k, v of a batch on the GPU, the forward call's results and, with d_out, the backward call's.  The tensors
    are views of wider buffers where `wide`; outputs start as NaN."""

    def __init__(self, batch, hq, hkv, d, dtype, seed=0, wide=False, q=None, k=None, v=None, d_out=None, scale=1.0):
        from paper_2604_26209_amd import binding as B
        self.B, self.batch, self.dims, self.dtype = B, batch, (hq, hkv, d), dtype
        n, td = batch.n, TD[dtype]
        self.layout = _layout(batch, hq, hkv, d, dtype)
        self.host = [x if x is not None else _normal(seed * 10 + i, (n, h, d), dtype, s) for i, (x, h, s) in
                     enumerate(((q, hq, scale), (k, hkv, scale), (v, hkv, 1.0)))]
        self.d_host = d_out if d_out is not None else _normal(seed * 10 + 5, (n, hq, d), dtype)
        self.nan = lambda *shape: torch.full(shape, float("nan"), dtype=td, device="cuda")

        def place(heads):
            """[n][heads][d] inside [n][heads + 3][d], from head 1 on"""
            return self.nan(n, heads + 3, d)[:, 1:1 + heads] if wide else self.nan(n, heads, d)

        self.q, self.k, self.v, self.dq, self.dk, self.dv = [place(h) for h in (hq, hkv, hkv, hq, hkv, hkv)]
        for t, x in zip((self.q, self.k, self.v), self.host):
            t.copy_(x)
        self.strides = B.hpd_finetune_strides(*[(x.stride(0) if wide else 0) for x in
                                                (self.q, self.k, self.v, self.dq, self.dk, self.dv)])
        self.out = self.nan(n, hq, d)
        self.lse = torch.full((hq, n), float("nan"), device="cuda")
        self.d_out = self.d_host.cuda()
        self.ws = [B.alloc_finetune_workspace(self.layout, b) for b in (False, True)]
        for w in self.ws:
            if w is not None:
                w.fill_(0xFF)

    def forward(self, stream=None):
        self.B.hpd_finetune_attention(self.layout, self.q, self.k, self.v, self.out, self.lse, self.ws[0], self.strides, stream)

    def backward(self, stream=None):
        self.B.hpd_finetune_attention_backward(self.layout, self.q, self.k, self.v, self.out, self.lse, self.d_out, self.dq,
                                               self.dk, self.dv, self.ws[1], self.strides, stream)

    def results(self):
        return [self.out, self.lse, self.dq, self.dk, self.dv]

    def check(self, label):
        hq, hkv, d = self.dims
        want = R.attention(self.batch, hq, hkv, *[R.to_numpy(x) for x in self.host], self.dtype, R.to_numpy(self.d_host),
                           R.to_numpy(self.out))
        for name in ("out", "lse", "dq", "dk", "dv"):
            R.check(getattr(self, name), *want[name], f"{label} {name}")


SHAPES = [  # hq, hkv, d, seed, sequences, prompt lengths, attributes, K_max
    (4, 4, 64, 1, 5, (0, 70), (0, 6), 7),
    (8, 2, 128, 2, 4, (20, 150), (0, 9), 12),
    (8, 1, 128, 3, 3, (100, 400), (2, 20), 32),
    (5, 1, 128, 4, 3, (0, 260), (0, 30), 5),
    (2, 2, 8, 5, 6, (0, 40), (0, 5), 4),
    (6, 2, 96, 6, 3, (10, 200), (1, 10), 16),
    (6, 1, 80, 7, 3, (0, 140), (1, 10), 16),
    (3, 3, 40, 8, 3, (0, 100), (0, 8), 9),
    (4, 2, 32, 9, 3, (0, 300), (0, 8), 9),
    (2, 1, 120, 10, 2, (120, 140), (0, 8), 9),
    (1, 1, 128, 11, 3, (500, 700), (10, 40), 16),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention_and_gradients(shape, dtype):
    hq, hkv, d, seed, n_seq, prompt, n_attr, k_max = shape
    batch = Batch.random(seed, n_seq, prompt, n_attr, k_max)
    print(f"attention {shape} {dtype}: {batch.len}", flush=True)
    r = Run(batch, hq, hkv, d, dtype, seed, wide=seed % 2 == 0)
    r.forward()
    r.backward()
    r.check(f"{shape} {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths_around_tiles(dtype, d):
    lens = [1, 2, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 160, 191, 192, 193, 255, 256, 257, 384, 385]
    batch = Batch([(n, [], []) for n in lens] + [(0, [], []), (0, [1], [0]), (0, [1], [3]), (0, [2, 1], [0, 4]), (127, [1], [1])],
                  4)
    r = Run(batch, 2, 1, d, dtype, 3)
    r.forward()
    r.backward()
    r.check(f"lengths {dtype} {d}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_values_hide_whole_tiles_of_keys(dtype):
    """Values of 150 tokens: the second value's first tokens do not see the last 120 of the first."""
    batch = Batch([(3, [1, 2, 1], [150, 150, 90]), (0, [1] * 3, [140, 10, 140])], 150)
    r = Run(batch, 2, 1, 128, dtype, 5)
    r.forward()
    r.backward()
    r.check(f"long values {dtype}")


@pytest.mark.parametrize("dtype, d", [("f32", 64), ("f32", 96), ("f32", 112), ("bf16", 24), ("bf16", 64), ("bf16", 80), ("bf16", 128)])
def test_tiles_cut_into_items(dtype, d):
    """One long sequence and few heads: a tile's rounds are shared by several workgroups.  Of the values of 600 tokens, the
    second's first ones see nothing of most of the first's, so neither do items of their tile."""
    from paper_2604_26209_amd import binding as B
    batch = Batch([(5, [1, 2, 1], [600, 600, 90]), (300, [1] * 4, [6, 0, 3, 7])], 600)
    r = Run(batch, 3, 1, d, dtype, 14, wide=True)
    counts = r.layout.counts()
    assert (counts[B.HPD_FTC_FORWARD_BYTES] > 0) == (dtype == "bf16")
    assert counts[B.HPD_FTC_BACKWARD_BYTES] > 8 * batch.n * 3 + 16
    r.forward()
    r.backward()
    r.check(f"items {dtype} {d}")
    first = [x.clone() for x in r.results()]
    r.forward()
    r.backward()
    assert all(torch.equal(a, b) for a, b in zip(first, r.results()))


@pytest.mark.parametrize("dtype, d", [("f32", 64), ("bf16", 64), ("bf16", 128), ("bf16", 96)])
def test_mask_of_the_gradients_row_by_row(dtype, d):
    """With the gradient of one query row per head, dv of every token is that row's weight times the row's gradient: exactly
    zero where the mask hides the token."""
    batch = Batch([(37, [2, 1, 3, 2, 4], [5, 0, 7, 3, 6]), (0, [1, 1, 1], [40, 3, 40]), (130, [1] * 12, [4] * 12)], 40)
    h = 8
    d_out = torch.zeros(batch.n, h, d)
    rows = {}
    for i, s in enumerate(batch.len):
        for j in range(h):
            rows[i, j] = s - 1 - (j * s // h)
            d_out[batch.off[i] + rows[i, j], j] = 1.0
    r = Run(batch, h, h, d, dtype, 6, d_out=d_out.to(TD[dtype]))
    r.forward()
    r.backward()
    r.check(f"rows {dtype} {d}")
    dv = R.to_numpy(r.dv)
    for (i, j), row in rows.items():
        got = dv[batch.off[i]:batch.off[i + 1], j, 0] != 0
        assert np.array_equal(got, batch.masks[i][row]), (i, j, row)


@pytest.mark.parametrize("scale", [0.0, 6.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_flat_and_peaked_scores(dtype, scale):
    """Equal scores: lse counts the visible tokens; scores of standard deviation 36: rows that one key dominates."""
    batch = Batch.random(12, 3, (30, 300), (2, 10), 9)
    r = Run(batch, 4, 2, 128, dtype, 7, scale=scale)
    r.forward()
    r.backward()
    r.check(f"scale {scale} {dtype}")
    if scale == 0.0:
        count = np.concatenate([m.sum(1) for m in batch.masks])
        assert np.allclose(R.to_numpy(r.lse), np.log(count), rtol=0, atol=4e-6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_far_below_and_above_zero(dtype):
    """A common offset of the scores, rising and falling along the keys, must cancel."""
    batch = Batch([(420, [2] * 4, [6] * 4), (90, [1], [9])], 9)
    d = 128
    q = torch.zeros(batch.n, 2, d)
    k = torch.zeros(batch.n, 1, d)
    q[:, 0, 0], q[:, 1, 0] = 16.0, -16.0
    k[:, 0, 0] = torch.linspace(-200, 200, batch.n).to(torch.bfloat16).float()
    r = Run(batch, 2, 1, d, dtype, 8, q=q.to(TD[dtype]), k=k.to(TD[dtype]))
    r.forward()
    r.backward()
    r.check(f"offsets {dtype}")


@pytest.mark.parametrize("hq, hkv, d", [(4, 2, 64), (2, 1, 128)])
def test_gradients_against_differences(hq, hkv, d):
    """Directional derivatives of sum(w * out), by central differences of the definition in 64 bits."""
    batch = Batch.random(21, 3, (5, 60), (1, 6), 6)
    r = Run(batch, hq, hkv, d, "f32", 9)
    r.forward()
    r.backward()
    host = [R.to_numpy(x) for x in r.host]
    w, eps = R.to_numpy(r.d_host), 1e-4
    bounds = R.attention(batch, hq, hkv, *host, "f32", w, R.to_numpy(r.out))
    rng = np.random.default_rng(0)
    for i, (x, name) in enumerate(zip(host, ("dq", "dk", "dv"))):
        for _ in range(2):
            step = rng.standard_normal(x.shape)
            value = []
            for sign in (1, -1):
                moved = list(host)
                moved[i] = x + sign * eps * step
                value.append((R.attention(batch, hq, hkv, *moved, "f32")["out"][0] * w).sum())
            want = (value[0] - value[1]) / (2 * eps)
            got = (R.to_numpy(getattr(r, name)) * step).sum()
            # (the differences themselves: a third derivative of order 1e2 times eps^2)
            assert abs(got - want) <= (bounds[name][1] * np.abs(step)).sum() + 1e-5 * (1 + abs(want)), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_calls_equal_bits_and_other_streams(dtype):
    batch = Batch.random(31, 5, (10, 300), (0, 12), 9)
    r = Run(batch, 8, 2, 128, dtype, 10)
    r.forward()
    r.backward()
    first = [x.clone() for x in r.results()]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for x in r.results():
        x.fill_(float("nan"))
    stream.wait_stream(torch.cuda.current_stream())
    r.forward(stream)
    r.backward(stream)
    torch.cuda.current_stream().wait_stream(stream)
    for a, b in zip(first, r.results()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype, d", [("f32", 64), ("bf16", 128), ("bf16", 96)])
def test_non_finite_values_stay_in_their_sequence(dtype, d):
    batch = Batch([(70, [1, 2], [3, 4]), (45, [1, 1], [5, 2]), (129, [2], [4])], 7)
    clean = Run(batch, 4, 2, d, dtype, 11)
    clean.forward()
    clean.backward()
    dirty = Run(batch, 4, 2, d, dtype, 11)
    sl = slice(batch.off[1], batch.off[2])
    for x, bad in ((dirty.q, float("nan")), (dirty.k, float("inf")), (dirty.v, float("nan")), (dirty.d_out, float("inf"))):
        x[sl] = bad
    dirty.forward()
    dirty.backward()
    for a, b in zip(clean.results(), dirty.results()):
        t = 1 if a is clean.lse else 0
        keep = torch.ones(batch.n, dtype=torch.bool, device="cuda")
        keep[sl] = False
        idx = torch.nonzero(keep)[:, 0]
        assert torch.equal(a.index_select(t, idx), b.index_select(t, idx))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_writes_stay_inside_the_outputs(dtype):
    """Outputs in wider buffers: what lies between the tokens keeps its contents."""
    batch = Batch.random(41, 4, (0, 150), (0, 9), 9)
    r = Run(batch, 4, 2, 128, dtype, 12, wide=True)
    r.forward()
    r.backward()
    for x in (r.dq, r.dk, r.dv):
        wide = x._base
        h = x.shape[1]
        assert bool(torch.isnan(wide[:, 0]).all()) and bool(torch.isnan(wide[:, 1 + h:]).all())
        assert bool(torch.isfinite(x).all())


def test_distances_beyond_32_bits():
    """Tokens 2^27 elements apart: offsets of 2^32 elements and more."""
    from paper_2604_26209_amd import binding as B
    batch = Batch([(30, [1, 2], [3, 2]), (3, [], [])], 4)
    n, hq, hkv, d, gap = batch.n, 2, 1, 128, 1 << 27
    assert n * gap > 1 << 32
    lay = _layout(batch, hq, hkv, d, "bf16")
    near = Run(batch, hq, hkv, d, "bf16", 13)
    near.forward()
    near.backward()
    buf = torch.empty(n * gap, dtype=torch.bfloat16, device="cuda")
    far = buf.view(n, gap)
    at = {"q": 0, "k": 1024, "v": 2048, "dq": 4096, "dk": 8192, "dv": 16384}
    view = {x: far[:, o:o + (hq if "q" in x else hkv) * d].view(n, -1, d) for x, o in at.items()}
    for x in ("q", "k", "v"):
        view[x].copy_(getattr(near, x))
    st = B.hpd_finetune_strides(gap, gap, gap, gap, gap, gap)
    out, lse = torch.empty_like(near.out), torch.empty_like(near.lse)
    B.hpd_finetune_attention(lay, view["q"], view["k"], view["v"], out, lse, near.ws[0], st)
    assert torch.equal(out, near.out) and torch.equal(lse, near.lse)
    B.hpd_finetune_attention_backward(lay, view["q"], view["k"], view["v"], out, lse, near.d_out, view["dq"], view["dk"],
                                      view["dv"], near.ws[1], st)
    for x in ("dq", "dk", "dv"):
        assert torch.equal(view[x], getattr(near, x)), x
    B.hpd_finetune_rotate(lay, 0, view["q"], view["k"], view["dq"], view["dk"], st)
    rq, rk = torch.empty_like(near.q), torch.empty_like(near.k)
    B.hpd_finetune_rotate(lay, 0, near.q, near.k, rq, rk)
    assert torch.equal(view["dq"], rq) and torch.equal(view["dk"], rk)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq, hkv, d", [(4, 2, 64), (32, 8, 128), (3, 1, 8), (6, 1, 80), (5, 5, 24), (2, 2, 40)])
def test_rotation_and_its_inverse(hq, hkv, d, dtype):
    from paper_2604_26209_amd import binding as B
    batch = Batch.random(51, 4, (0, 200), (0, 12), 30)  # (gaps: fewer tokens than positions)
    more = Batch([(700, [], []), (300, [1], [3])], 4)
    for b in (batch, more):
        lay = _layout(b, hq, hkv, d, dtype, 500000.0)
        q, k = _normal(1, (b.n, hq, d), dtype), _normal(2, (b.n, hkv, d), dtype)
        for inverse in (0, 1):
            qd, kd = q.cuda(), k.cuda()
            qo, ko = torch.full_like(qd, float("nan")), torch.full_like(kd, float("nan"))
            B.hpd_finetune_rotate(lay, inverse, qd, kd, qo, ko)
            for x, y in ((q, qo), (k, ko)):
                x64 = R.to_numpy(x)
                want = R.rotate(b.pos, 500000.0, x64, bool(inverse))
                half = d // 2
                pair = np.abs(x64[..., :half]) + np.abs(x64[..., half:])
                # cos, sin rounded to fp32, two products and a sum; then the output's rounding
                bound = 4 * R.U32 * np.concatenate([pair, pair], -1) + R.U[dtype] * np.abs(want)
                R.check(y, want, bound, f"rotate {hq}/{hkv}x{d} {dtype}")
            B.hpd_finetune_rotate(lay, inverse, qd, kd, qd, kd)  # in place
            assert torch.equal(qd, qo) and torch.equal(kd, ko)


def test_refusals_of_device_layouts():
    from paper_2604_26209_amd import binding as B
    batch = Batch([(9, [1], [2])], 4)
    r = Run(batch, 4, 2, 64, "bf16", 1)

    def status(f, *a):
        with pytest.raises(B.HpdError) as e:
            f(*a)
        return e.value.status
    off = r.q.data_ptr() + 2
    small, odd = B.hpd_finetune_strides(q=4 * 64 - 8), B.hpd_finetune_strides(v=2 * 64 + 4)
    fwd = [r.layout, r.q, r.k, r.v, r.out, r.lse, r.ws[0], None]
    bwd = [r.layout, r.q, r.k, r.v, r.out, r.lse, r.d_out, r.dq, r.dk, r.dv, r.ws[1], None]
    rot = [r.layout, 0, r.q, r.k, r.dq, r.dk, None]
    for f, args, pointers in ((B.hpd_finetune_attention, fwd, range(1, 6)),
                              (B.hpd_finetune_attention_backward, bwd, range(1, 11)),
                              (B.hpd_finetune_rotate, rot, range(2, 6))):
        for i in pointers:
            for bad in (None, off):
                assert status(f, *[bad if j == i else a for j, a in enumerate(args)]) == B.HPD_E_INVALID, (f.__name__, i)
        for bad in (small, odd):
            assert status(f, *args[:-1], bad) == B.HPD_E_INVALID
    empty = _layout(Batch([(0, [], [])], 3), 4, 2, 64, "bf16")  # no tokens: nothing to do, whatever the tensors are
    B.hpd_finetune_rotate(empty, 0, None, None, None, None)
    B.hpd_finetune_attention(empty, None, None, None, None, None)
    B.hpd_finetune_attention_backward(empty, *[None] * 9)


def test_forward_and_backward_in_a_graph():
    """A captured step, replayed with other inputs in the same tensors and eager work in between."""
    batch = Batch.random(61, 4, (20, 250), (1, 9), 9)
    r = Run(batch, 8, 2, 128, "bf16", 14)
    r.forward()
    r.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.forward()
        r.backward()
    for turn in range(3):
        r.q.copy_(_normal(100 + turn, tuple(r.q.shape), "bf16"))
        r.d_out.copy_(_normal(200 + turn, tuple(r.d_out.shape), "bf16"))
        r.forward()
        r.backward()
        want = [x.clone() for x in r.results()]
        for x in r.results():
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, r.results()):
            assert torch.equal(a, b), turn


# ---------------------------------------------------------------------------------------------
# log probabilities
# ---------------------------------------------------------------------------------------------
def _logits(seed, rows, vocab, stride, dtype, scale=2.5):
    """On the GPU: [rows][vocab] inside [rows][stride] behind one more element (rows on any alignment)."""
    buf = torch.full((rows * stride + 1,), float("nan"), dtype=TD[dtype], device="cuda")
    x = buf[1:].view(rows, stride)[:, :vocab]
    x.copy_(_normal(seed, (rows, vocab), dtype, scale))
    return x


def _run_logprobs(x, target, top, entropy=True):
    from paper_2604_26209_amd import binding as B
    rows, vocab = x.shape
    dt = _dtype("f32" if x.dtype == torch.float32 else "bf16")
    n = B.hpd_token_logprobs_workspace(dt, rows, vocab, top)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None
    res = [torch.full((rows,), float("nan"), device="cuda") for _ in range(3)]
    ids = torch.full((rows, top), -7, dtype=torch.int32, device="cuda")
    vals = torch.full((rows, top), float("nan"), device="cuda")
    B.hpd_token_logprobs(dt, rows, vocab, x.stride(0), x, target, top, res[0], res[1], res[2], ids if top else None,
                         vals if top else None, ws)
    return (*res, ids, vals)


def _sum_error(x64, lse):
    """What log(sum of exponentials) may be off by: every exponential by the rounding of its argument (twice, one more time
    per change of the reference point) and of its own, the sum by its terms per lane."""
    vocab = x64.shape[1]
    p = np.exp(x64 - lse[:, None])
    d = np.where(p > 0, np.abs(x64 - np.max(x64, axis=1, keepdims=True)), 0.0)
    return R.U32 * (3 * (p * d).sum(1) + vocab / 64 + 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, pad, top", [
    (1, 1, 0, 1), (3, 5, 0, 5), (7, 63, 1, 50), (9, 64, 0, 64), (5, 500, 3, 8), (64, 513, 0, 1), (33, 2047, 0, 64),
    (6, 2049, 5, 20), (11, 4096, 0, 0), (300, 8200, 7, 5), (4, 33333, 0, 64), (1, 150001, 1, 20), (1100, 4200, 0, 3),
    (2, 1000003, 0, 33)])
def test_log_probabilities(rows, vocab, pad, top, dtype):
    x = _logits(vocab + top, rows, vocab, vocab + pad, dtype)
    rng = np.random.default_rng(vocab)
    target = rng.integers(0, vocab, rows)
    target[::5] = rng.choice([-1, vocab, -2 ** 31, 2 ** 31 - 1], target[::5].shape)
    logprob, lse, ent, ids, vals = _run_logprobs(x, torch.from_numpy(target.astype(np.int32)).cuda(), top)
    x64 = R.to_numpy(x)
    w_logprob, w_lse, w_ent, w_ids, w_vals = R.logprobs(x64, target, top)
    e = _sum_error(x64, w_lse) + 2 * R.U32 * np.abs(w_lse)
    R.check(lse, w_lse, e, "lse")
    R.check(logprob, w_logprob, np.where(w_logprob != 0, e + 2 * R.U32 * np.abs(w_logprob), 0.0), "log probability")
    p = np.exp(x64 - w_lse[:, None])
    spread = (p * np.abs(x64 - x64.max(1, keepdims=True))).sum(1)
    R.check(ent, w_ent, 3 * e * (1 + spread), "entropy")
    assert np.array_equal(ids.cpu().numpy(), w_ids)
    R.check(vals, w_vals, e[:, None] + 2 * R.U32 * np.abs(w_vals), "alternatives")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [70, 3000, 40000])
def test_order_of_alternatives(vocab, dtype):
    """Equal logits: the lowest index first; rising and falling rows; negative zero; few values; -infinity among them."""
    up = torch.arange(vocab, dtype=torch.float32)
    rows = [torch.zeros(vocab), torch.where(up % 2 == 0, 0.0, -0.0), up / 64, -up / 64, (up % 7), -(up % 5),
            torch.where(up % 3 == 1, 1.0, -float("inf")), torch.where(up == vocab - 1, 2.0, -float("inf"))]
    x = torch.stack(rows).to(TD[dtype]).cuda()
    target = torch.full((len(rows),), vocab - 1, dtype=torch.int32, device="cuda")
    _, _, _, ids, vals = _run_logprobs(x, target, 64)
    x64 = R.to_numpy(x)
    _, lse, _, w_ids, w_vals = R.logprobs(x64, np.full(len(rows), vocab - 1), 64)
    assert np.array_equal(ids.cpu().numpy(), w_ids)
    got = R.to_numpy(vals)
    assert np.array_equal(np.isneginf(got), np.isneginf(w_vals))
    fin = np.isfinite(w_vals)
    assert np.abs(got[fin] - w_vals[fin]).max() <= 1e-6 * (vocab / 64 + np.abs(w_vals[fin]).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 5000, 70000])
def test_rows_with_masked_and_non_finite_logits(vocab, dtype):
    from paper_2604_26209_amd import binding as B
    inf, lowest = float("inf"), torch.finfo(TD[dtype]).min
    x = _normal(5, (8, vocab), dtype)
    x[0] = -inf                         # nothing left
    x[1] = -inf
    x[1, vocab // 2] = 3.0              # one token left
    x[2, 1::2] = -inf
    x[3] = lowest                       # all of the type's lowest value: equal
    x[4, : vocab - 1] = lowest          # ... or excluded by it
    x[5, vocab - 1] = float("nan")
    x[6, 0] = inf
    x[7, ::3] = lowest
    x = x.cuda()
    target = torch.tensor([3, vocab // 2, 1, 4, vocab - 1, 2, 2, 0], dtype=torch.int32, device="cuda")
    logprob, lse, ent, ids, vals = [R.to_numpy(t) for t in _run_logprobs(x, target, 4)]
    assert lse[0] == -inf and logprob[0] == -inf and ent[0] == 0 and np.array_equal(ids[0], range(4)) and (vals[0] == -inf).all()
    assert abs(lse[1] - 3) < 1e-6 and abs(logprob[1]) < 1e-6 and abs(ent[1]) < 1e-6 and ids[1, 0] == vocab // 2
    assert logprob[2] == -inf and np.isfinite(ent[2]) and np.isfinite(vals[2]).all()
    assert abs(logprob[3] + np.log(vocab)) < 1e-4 and abs(ent[3] - np.log(vocab)) < 1e-4
    assert abs(logprob[4]) < 1e-6 and abs(ent[4]) < 1e-6
    for row in (5, 6):
        assert np.isnan(lse[row]) and np.isnan(logprob[row]) and np.isnan(ent[row])
        assert ((ids[row] >= 0) & (ids[row] < vocab)).all()
    w = R.logprobs(R.to_numpy(x)[7:], np.array([0]), 4)
    assert abs(lse[7] - w[1][0]) < 1e-5 and abs(ent[7] - w[2][0]) < 1e-4 and np.array_equal(ids[7], w[3][0])
    # gradients: no NaN where there is none
    rows = x.shape[0]
    l32, e32 = [torch.from_numpy(t).float().cuda() for t in (lse, ent)]
    d = torch.full_like(x, 7.0)
    ones = torch.ones(rows, device="cuda")
    B.hpd_token_logprobs_backward(_dtype(dtype), rows, vocab, vocab, x, target, l32, e32, ones, ones, d, vocab)
    d = R.to_numpy(d)
    assert (d[0] == 0).all() and np.abs(d[1]).max() <= 1e-5
    assert np.isfinite(d[[2, 3, 4, 7]]).all() and np.isnan(d[5]).all()
    assert (d[2, 3::2] == 0).all() and d[2, 1] == 1.0  # excluded tokens: only the target's own term


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, pad, d_pad", [(1, 1, 0, 0), (3, 7, 1, 0), (5, 500, 0, 3), (17, 2048, 0, 0),
                                                     (6, 8191, 2, 1), (40, 8193, 0, 0), (9, 50021, 1, 2)])
@pytest.mark.parametrize("with_entropy", [False, True])
def test_gradient_of_log_probabilities(rows, vocab, pad, d_pad, with_entropy, dtype):
    from paper_2604_26209_amd import binding as B
    x = _logits(vocab, rows, vocab, vocab + pad, dtype)
    rng = np.random.default_rng(vocab)
    target = rng.integers(0, vocab, rows)
    target[1::4] = -1
    x64 = R.to_numpy(x)
    _, lse, ent, _, _ = R.logprobs(x64, target, 0)
    g, h = rng.standard_normal(rows), rng.standard_normal(rows) * with_entropy
    f = lambda a: torch.from_numpy(np.asarray(a)).float().cuda()
    lse32, ent32, g32, h32 = f(lse), f(ent), f(g), f(h)
    buf = torch.full((rows, vocab + d_pad), 7.0, dtype=TD[dtype], device="cuda")
    t32 = torch.from_numpy(target.astype(np.int32)).cuda()
    args = (t32, lse32, ent32 if with_entropy else None, g32, h32 if with_entropy else None)
    B.hpd_token_logprobs_backward(_dtype(dtype), rows, vocab, x.stride(0), x, *args, buf, vocab + d_pad)
    # from the 32-bit numbers that the call is given
    g, h, lse, ent = [R.to_numpy(t) for t in (g32, h32, lse32, ent32)]
    lp = x64 - lse[:, None]
    p = np.exp(lp)
    has = target >= 0
    gt = np.where(has, g, 0.0)[:, None]
    want = -gt * p - h[:, None] * p * (lp + ent[:, None])
    want[has, target[has]] += g[has]
    part = p * (np.abs(gt) + np.abs(h)[:, None] * (np.abs(lp) + ent[:, None]))
    at = np.zeros_like(want)
    at[has, target[has]] = np.abs(g[has])
    # the argument's rounding, the exponential, the factors and their sum; then the output's rounding
    bound = R.U32 * (part * (4 * np.abs(lp) + 16) + 4 * at) + R.U[dtype] * np.abs(want) * (1 + 2 ** -6) + 2.0 ** -126
    R.check(buf[:, :vocab], want, bound, "gradient")
    assert bool((buf[:, vocab:] == 7.0).all())
    # in place
    B.hpd_token_logprobs_backward(_dtype(dtype), rows, vocab, x.stride(0), x, *args, x, x.stride(0))
    assert torch.equal(x, buf[:, :vocab])


def test_gradient_of_log_probabilities_against_differences():
    from paper_2604_26209_amd import binding as B
    rows, vocab, eps = 4, 777, 1e-5
    x = _logits(3, rows, vocab, vocab, "f32")
    target = np.array([5, 0, -1, 776])
    t32 = torch.from_numpy(target.astype(np.int32)).cuda()
    _, lse, ent, _, _ = _run_logprobs(x, t32, 0)
    rng = np.random.default_rng(1)
    g, h = rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
    d = torch.empty(rows, vocab, device="cuda")
    B.hpd_token_logprobs_backward(B.HPD_F32, rows, vocab, vocab, x, t32, lse, ent, torch.from_numpy(g).cuda(),
                                  torch.from_numpy(h).cuda(), d, vocab)
    x64 = R.to_numpy(x)
    for seed in range(4):
        step = np.random.default_rng(seed).standard_normal(x64.shape)
        f = []
        for sign in (1, -1):
            lp, _, en, _, _ = R.logprobs(x64 + sign * eps * step, target, 0)
            f.append((g * lp + h * en).sum())
        want = (f[0] - f[1]) / (2 * eps)
        assert abs((R.to_numpy(d) * step).sum() - want) <= 1e-4 * (1 + abs(want))


def test_logit_rows_beyond_32_bits():
    from paper_2604_26209_amd import binding as B
    rows, vocab, stride = 5, 3001, 1 << 30
    far = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").view(rows, stride)[:, :vocab]
    near = _normal(4, (rows, vocab), "bf16").cuda()
    far.copy_(near)
    target = torch.arange(rows, dtype=torch.int32, device="cuda")
    a, b = _run_logprobs(near, target, 6), _run_logprobs(far, target, 6)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    ones = torch.ones(rows, device="cuda")
    d = torch.empty_like(near)
    B.hpd_token_logprobs_backward(B.HPD_BF16, rows, vocab, vocab, near, target, a[1], a[2], ones, ones, d, vocab)
    B.hpd_token_logprobs_backward(B.HPD_BF16, rows, vocab, stride, far, target, a[1], a[2], ones, ones, far, stride)
    assert torch.equal(d, far)


def test_log_probabilities_in_a_graph():
    from paper_2604_26209_amd import binding as B
    rows, vocab, top = 6, 60000, 9
    x = _normal(6, (rows, vocab), "bf16").cuda()
    target = torch.arange(rows, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.hpd_token_logprobs_workspace(B.HPD_BF16, rows, vocab, top), dtype=torch.uint8, device="cuda")
    res = [torch.empty(rows, device="cuda") for _ in range(3)]
    ids, vals = torch.empty(rows, top, dtype=torch.int32, device="cuda"), torch.empty(rows, top, device="cuda")
    d, ones = torch.empty_like(x), torch.ones(rows, device="cuda")

    def step():
        B.hpd_token_logprobs(B.HPD_BF16, rows, vocab, vocab, x, target, top, *res, ids, vals, ws)
        B.hpd_token_logprobs_backward(B.HPD_BF16, rows, vocab, vocab, x, target, res[1], res[2], ones, ones, d, vocab)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        x.copy_(_normal(300 + turn, (rows, vocab), "bf16"))
        step()
        want = [t.clone() for t in (*res, ids, vals, d)]
        for t in (*res, vals, d):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (*res, ids, vals, d)):
            assert torch.equal(a, b), turn
