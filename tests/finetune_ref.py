"""Plain 64-bit forms of the fine-tuning operators, written from their definitions, with bounds on the
error that the roundings of a 32-bit (or bf16) computation may leave.  TEST INFRASTRUCTURE ONLY.

Roundings counted: u = half a step of the type (bf16 2^-8, fp32 2^-24), relative to the value.  Under
bf16 the weights p and the scores' gradients ds are rounded once before the second products and
every output once; sums are in fp32: a sum of n terms is off by at most n * 2^-24 of the sum of
their magnitudes, and a score that is off by e changes its weight by the factor exp(e)."""
import numpy as np
import torch

from oracle import finetune_mask as FM

U32 = 2.0 ** -24
U = {"f32": U32, "bf16": 2.0 ** -8}


class Batch:
    """Lengths of packed training sequences with their positions and masks from the oracle."""

    def __init__(self, seqs, k_max):
        """seqs: (prompt_len, attr_lens, value_lens) per sequence"""
        self.seqs, self.k_max = seqs, k_max
        self.prompt_len = np.array([s[0] for s in seqs], np.int32)
        self.attr_ptr = np.cumsum([0] + [len(s[1]) for s in seqs]).astype(np.int32)
        self.attr_len = np.array([a for s in seqs for a in s[1]], np.int32)
        self.value_len = np.array([v for s in seqs for v in s[2]], np.int32)
        self.len = [int(s[0] + sum(s[1]) + sum(s[2])) for s in seqs]
        self.off = np.cumsum([0] + self.len)
        self.n = int(self.off[-1])
        self.pos = np.concatenate([FM.finetune_position_ids(p, a, v, k_max) for p, a, v in seqs]
                                  or [np.zeros(0, np.int64)]).astype(np.int64)
        self.masks = [self.mask(i) for i in range(len(seqs))]

    def mask(self, i):
        p, a, v = self.seqs[i]
        kind, attr, k = FM.finetune_tokens(p, a, v)
        s = len(kind)
        if s <= 200:  # the oracle's loops
            return FM.finetune_mask(p, a, v).astype(bool)
        # the same three rules on whole arrays
        later = np.arange(s)[None, :] > np.arange(s)[:, None]
        value = kind == FM.KIND_VALUE
        name_sees_value = (kind == FM.KIND_ATTR)[:, None] & value[None, :]
        not_yet = value[:, None] & value[None, :] & (attr[None, :] < attr[:, None]) & (k[None, :] > k[:, None])
        return ~(later | name_sees_value | not_yet)

    @staticmethod
    def random(seed, n_seq, prompt=(0, 60), n_attr=(0, 6), k_max=7):
        rng = np.random.default_rng(seed)
        seqs = []
        for _ in range(n_seq):
            m = int(rng.integers(n_attr[0], n_attr[1] + 1))
            seqs.append((int(rng.integers(prompt[0], prompt[1] + 1)), rng.integers(1, 5, m).tolist(),
                         rng.integers(0, k_max + 1, m).tolist()))
        return Batch(seqs, k_max)


def attention(batch, hq, hkv, q, k, v, dtype, d_out=None, out=None):
    """q [N][hq][D], k, v [N][hkv][D] (numpy float64, the values of the type).  Returns a dict of
    (value, bound) pairs: out, lse, and with d_out and out (the forward result that the backward
    call is given) dq, dk, dv."""
    n, _, d = q.shape
    g, u, scale = hq // hkv, U[dtype], 1.0 / np.sqrt(d)
    low = u if dtype == "bf16" else 0.0  # rounding of p and ds before the second products
    res = {x: (np.zeros(s), np.zeros(s)) for x, s in
           (("out", (n, hq, d)), ("lse", (hq, n)), ("dq", (n, hq, d)), ("dk", (n, hkv, d)), ("dv", (n, hkv, d)))}
    for i, s in enumerate(batch.len):
        sl = slice(batch.off[i], batch.off[i] + s)
        if s == 0:
            continue
        gamma = (s + d + 32) * U32  # sums of s or d terms, exponentials, rescaling
        for h in range(hq):
            c = h // g
            qh, kh, vh = q[sl, h], k[sl, c], v[sl, c]
            score = np.where(batch.masks[i], qh @ kh.T * scale, -np.inf)
            # what a score may be off by; its exponential is then off by that factor
            es = gamma * np.where(batch.masks[i], np.abs(qh) @ np.abs(kh).T * scale + np.abs(score), 0.0)
            top = score.max(1, keepdims=True)
            p = np.exp(score - top)
            total = p.sum(1, keepdims=True)
            p /= total
            lse = (top + np.log(total))[:, 0]
            res["lse"][0][h, sl] = lse
            elp = (p * es).sum(1)
            res["lse"][1][h, sl] = elp + 2 * gamma + 4 * U32 * np.abs(lse)
            o = p @ vh
            # relative error of a normalised weight: its score's, the row's sum's, the rounding
            ew = p * (es + elp[:, None] + 2 * gamma + low)
            res["out"][0][sl, h] = o
            res["out"][1][sl, h] = ew @ np.abs(vh) * (1 + 2 ** -6) + u * np.abs(o) + 1e-30
            if d_out is None:
                continue
            do = d_out[sl, h]
            delta = (do * o).sum(1)
            e_delta = np.abs(do * (out[sl, h] - o)).sum(1) + gamma * np.abs(do * o).sum(1)
            dp = do @ vh.T
            e_dp = gamma * (np.abs(do) @ np.abs(vh).T)
            ep = p * (es + 4 * U32 * np.abs(lse)[:, None] + gamma)  # p = exp(s - lse) in fp32
            ds = p * (dp - delta[:, None]) * scale
            e_ds = (ep * np.abs(dp - delta[:, None]) + p * (e_dp + e_delta[:, None])) * scale
            e_ds = (e_ds + (low + 4 * gamma) * np.abs(ds)) * (1 + 2 ** -6)
            ep = ep + (low + gamma) * p
            res["dq"][0][sl, h] = ds @ kh
            res["dq"][1][sl, h] = e_ds @ np.abs(kh)
            res["dk"][0][sl, c] += ds.T @ qh
            res["dk"][1][sl, c] += e_ds.T @ np.abs(qh)
            res["dv"][0][sl, c] += p.T @ do
            res["dv"][1][sl, c] += ep.T @ np.abs(do) * (1 + 2 ** -6)
    if d_out is not None:
        for x in ("dq", "dk", "dv"):
            res[x] = (res[x][0], res[x][1] + (u + g * U32) * np.abs(res[x][0]) + 1e-30)
    return res


def rotate(pos, base, x, inverse=False):
    """x [N][H][D] float64"""
    half = x.shape[-1] // 2
    theta = np.array([base ** (-m / half) for m in range(half)])
    ang = (-1 if inverse else 1) * pos[:, None].astype(np.float64) * theta
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def logprobs(x, target, top):
    """x [n][V] float64 (values of the type), target int [n].  Returns (logprob, lse, entropy, ids, values)."""
    n, v = x.shape
    with np.errstate(all="ignore"):
        m = x.max(1)
        none = np.isneginf(m)
        e = np.exp(x - np.where(none, 0.0, m)[:, None])
        s = e.sum(1)
        lse = np.where(none, -np.inf, m + np.log(s))
        p = e / np.where(none, 1.0, s)[:, None]
        lp = np.where(none[:, None], -np.inf, x - lse[:, None])
        h = -np.where(p > 0, p * np.log(np.where(p > 0, p, 1.0)), 0.0).sum(1)
        has = (target >= 0) & (target < v)
        logprob = np.where(has, lp[np.arange(n), np.where(has, target, 0)], 0.0)
        ids = np.argsort(-x, axis=1, kind="stable")[:, :top]
    return logprob, lse, h, ids, np.take_along_axis(lp, ids, 1)


def to_numpy(t):
    return t.detach().double().cpu().numpy()


def check(got, want, bound, label):
    got = to_numpy(got) if torch.is_tensor(got) else got
    assert np.isfinite(got).all(), f"{label}: not finite"
    over = np.abs(got - want) > bound
    if over.any():
        at = tuple(int(x) for x in np.argwhere(over)[0])
        raise AssertionError(f"{label}: {int(over.sum())} of {over.size} off, first at {at}: {got[at]!r} for {want[at]!r}, "
                             f"bound {bound[at]:.3e}")
