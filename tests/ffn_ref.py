"""The feed-forward block and the vocabulary head in 64 bits, and bounds of what their kernels' arithmetic may be off.

Rounding: a value rounded to a type is off by half a step, eps / 2 of it.  A sum of K products in fp32, in any
order, is off by at most K 2^-23 times the sum of their magnitudes (a multiplication and an addition each, half a
step 2^-24).  fp32 functions (exp, erf, division) are taken as good to FUNC relative to their largest factor, and act's
slope is at most 1.13 in magnitude, act(x) at most |x|."""
import math

import torch

U = 2.0 ** -23
FUNC = 2.0 ** -19
SLOPE = 1.2


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def act(g, name):
    """The activation and its derivative."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        c = 0.5 * torch.special.erfc(-g * math.sqrt(0.5))
        return g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    w = math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3)
    s = torch.sigmoid(w)
    return g * s, s + g * s * (1 - s) * math.sqrt(8 / math.pi) * (1 + 3 * 0.044715 * g * g)


def product(a, b, error_a=None):
    """a b^T and a bound of its error, for a's own error."""
    c = a @ b.T
    magnitude = a.abs() @ b.abs().T
    error = a.shape[1] * U * magnitude
    if error_a is not None:
        error = error + error_a @ b.abs().T * (1 + a.shape[1] * U)
    return c, error


def ffn(x, wg, wu, wd, name, dtype):
    """(value, bound) of out, gate and up; inputs in 64 bits, h held as dtype."""
    eps = half_step(dtype)
    g, eg = product(x, wg)
    u, eu = product(x, wu)
    a, _ = act(g, name)
    h = a * u
    eh = (SLOPE * eg + FUNC * g.abs()) * (u.abs() + eu) + a.abs() * eu
    eh = eh + eps * (h.abs() + eh)
    out, eo = product(h, wd, eh)
    return [(v, e + eps * (v.abs() + e)) for v, e in ((out, eo), (g, eg), (u, eu))]


def ffn_grad(x, wg, wu, wd, g, u, d_out, name, dtype):
    """(value, bound) of dx, dwg, dwu, dwd for the given g and u."""
    eps = half_step(dtype)
    a, slope = act(g, name)
    dh, edh = product(d_out, wd.T)
    h = a * u
    eh = FUNC * (g * u).abs()
    eh = eh + eps * (h.abs() + eh)
    dg, du = dh * u * slope, dh * a
    # (slope: its terms are at most 1 + |g|)
    edg = edh * u.abs() * SLOPE + FUNC * (dh * u).abs() * (1 + g.abs())
    edu = edh * a.abs() + FUNC * (dh * g).abs()
    edg, edu = edg + eps * (dg.abs() + edg), edu + eps * (du.abs() + edu)
    dx, ex = product(torch.cat([dg, du], 1), torch.cat([wg, wu], 0).T, torch.cat([edg, edu], 1))
    dwg, ewg = product(dg.T, x.T, edg.T)
    dwu, ewu = product(du.T, x.T, edu.T)
    dwd, ewd = product(h.T, d_out.T, eh.T)
    return [(v, e + eps * (v.abs() + e)) for v, e in ((dx, ex), (dwg, ewg), (dwu, ewu), (dwd.T, ewd.T))]


def head(x, w, targets):
    """(value, bound) of logprob, lse and entropy."""
    logits, e = product(x, w)
    return logprobs(logits, targets, e)


def logprobs(logits, targets, e):
    n, v = logits.shape
    lse = torch.logsumexp(logits, 1)
    lp = logits - lse[:, None]
    p = lp.exp()
    far = torch.where(p > 0, lp, 0.0)
    entropy = -(p * far).sum(1)
    has = (targets >= 0) & (targets < v)
    at = torch.where(has, targets, 0).long()[:, None]
    logprob = torch.where(has, lp.gather(1, at)[:, 0], 0.0)
    # a term of the sum: its logit, the rounding of the difference to the maximum and of its scaling, the exponential;
    # and the additions on its way (in a lane at most 64, over lanes, waves and tiles at most 30 and one per 64 tiles of 64)
    top = logits.amax(1, keepdim=True)
    d = (logits - top).clamp(min=-200.0)
    term = e + 2.0 ** -22 * d.abs() + U * (100 + v / 4096)
    e_sum = (p * term).sum(1)
    e_log = e_sum + U * (1 + (lse - top[:, 0]).abs())
    e_lse = e_log + U * lse.abs()
    e_logprob = torch.where(has, e_log + e.gather(1, at)[:, 0] + U * (logits.gather(1, at)[:, 0] - top[:, 0]).abs() + U * logprob.abs(), 0.0)
    # entropy = log s - t / s, t a sum of e^d d
    e_entropy = e_log + (p * (term * (1 + 2 * d.abs()) + e)).sum(1) + e_sum * (p * d.abs()).sum(1) + U * (1 + entropy.abs())
    return [(logprob, e_logprob), (lse, e_lse), (entropy, e_entropy)]


def head_grad(x, w, targets, lse, entropy, g_logprob, g_entropy, dtype):
    """(value, bound) of d_hidden and d_weight for the given lse and entropy."""
    eps = half_step(dtype)
    logits, e = product(x, w)
    n, v = logits.shape
    has = (targets >= 0) & (targets < v)
    g = torch.where(has, g_logprob, 0.0)[:, None] if g_logprob is not None else torch.zeros((n, 1), dtype=torch.float64, device=x.device)
    ge = g_entropy[:, None] if g_entropy is not None else torch.zeros_like(g)
    H = entropy[:, None] if g_entropy is not None else torch.zeros_like(g)
    lp = logits - lse[:, None]
    p = lp.exp()
    hot = torch.zeros_like(p).scatter_(1, torch.where(has, targets, 0).long()[:, None], 1.0) * has[:, None]
    factor = g + ge * (lp + H)
    d = g * hot - p * factor
    e_lp = e + U * lp.abs()
    e_factor = ge.abs() * (e_lp + U * (lp + H).abs()) + U * factor.abs() + U * (ge * (lp + H)).abs()
    ed = p * (factor.abs() * (1.01 * e_lp + U * (2 + lp.abs())) + e_factor) + U * (g * hot).abs() + U * d.abs()
    ed = ed + eps * (d.abs() + ed)
    dx, ex = product(d, w.T, ed)
    dw, ew = product(d.T, x.T, ed.T)
    return [(a, b + eps * (a.abs() + b)) for a, b in ((dx, ex), (dw, ew))]


def check(got, want, what):
    value, bound = want
    got = got.double()
    assert got.shape == value.shape, what
    off = (got - value).abs()
    bad = ~(off <= bound + 1e-37)
    if bad.any():
        i = tuple(int(k) for k in torch.nonzero(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} are off, first {i}: {got[i].item()} for "
                             f"{value[i].item()}, allowed {bound[i].item()}")


# ---------------------------------------------------------------------------
# Bounds by likelihood: a long contraction's worst case would let a lost element through.  Roundings are taken as independent of each
# other and of the signs of what they are multiplied with.  A value's rounding, at most half a step, has a standard deviation of
# half a step / sqrt 3; a sum of K products rounds K times (an addition each, a product goes in unrounded or with a rounding that is
# small next to the sum's), each time at most 2^-24 of a partial sum, which on its way is of the size of the end result c
# or of sqrt(sum a^2 b^2), what a sum of random signs has.  Errors of fp32 functions, FUNC, have the signs of what they are
# multiplied with.  A result may be LIKELY deviations off (7: 3e-12 of normal values are, of 4e7 in a test) and its own last rounding.
# ---------------------------------------------------------------------------
LIKELY = 7.0


def likely_product(a, b, deviation_a=None):
    """a b^T and the standard deviation of its error, for that of a's elements."""
    c = a @ b.T
    squares = b.T ** 2
    variance = a.shape[1] * 2.0 ** -48 * ((a ** 2) @ squares + c ** 2)
    if deviation_a is not None:
        variance = variance + (deviation_a ** 2) @ squares
    return c, variance.sqrt()


def _likely(v, deviation, eps):
    e = LIKELY * deviation
    return v, e + eps * (v.abs() + e)


def _norm(*terms):
    return sum(t ** 2 for t in terms).sqrt()


def likely_ffn(x, wg, wu, wd, name, dtype):
    """(value, bound) of out, gate and up."""
    eps = half_step(dtype)
    g, sg = likely_product(x, wg)
    u, su = likely_product(x, wu)
    a, _ = act(g, name)
    h = a * u
    sh = _norm(SLOPE * sg * u, a * su, FUNC * g * u, eps / math.sqrt(3) * h)
    return [_likely(v, s, eps) for v, s in (likely_product(h, wd, sh), (g, sg), (u, su))]


def likely_ffn_grad(x, wg, wu, wd, g, u, d_out, name, dtype):
    """(value, bound) of dx, dwg, dwu, dwd for the given g and u."""
    eps = half_step(dtype)
    step = eps / math.sqrt(3)
    a, slope = act(g, name)
    dh, sdh = likely_product(d_out, wd.T)
    h, dg, du = a * u, dh * u * slope, dh * a
    sh = _norm(FUNC * g * u, step * h)
    sdg = _norm(sdh * u * SLOPE, FUNC * dh * u * (1 + g.abs()), step * dg)
    sdu = _norm(sdh * a, FUNC * dh * g, step * du)
    dx = likely_product(torch.cat([dg, du], 1), torch.cat([wg, wu], 0).T, torch.cat([sdg, sdu], 1))
    dwg, dwu = likely_product(dg.T, x.T, sdg.T), likely_product(du.T, x.T, sdu.T)
    dwd = likely_product(h.T, d_out.T, sh.T)
    return [_likely(v, s, eps) for v, s in (dx, dwg, dwu, (dwd[0].T, dwd[1].T))]


def likely_head(x, w, targets):
    """(value, bound) of logprob, lse and entropy."""
    logits, s = likely_product(x, w)
    return logprobs(logits, targets, LIKELY * s)


def likely_head_grad(x, w, targets, g_logprob, dtype):
    """(value, bound) of d_hidden and d_weight, no entropy: with an lse that the same kernels made."""
    eps = half_step(dtype)
    logits, s = likely_product(x, w)
    lse = torch.logsumexp(logits, 1, keepdim=True)
    p = (logits - lse).exp()
    at = targets.long()[:, None]
    hot = torch.zeros_like(p).scatter_(1, at, 1.0)
    d = g_logprob[:, None] * (hot - p)
    # p by its logit's error and by the lse's: the mean of the logits' by their p, its sum's and its own rounding; the product is rounded
    e_lse = (p * s).sum(1, keepdim=True) + U * (100 + w.shape[0] / 4096) + U * lse.abs()
    sd = _norm(g_logprob[:, None] * p * (s + e_lse + U * (2 + (logits - lse).abs())), eps / math.sqrt(3) * d, U * g_logprob[:, None] * hot)
    return [_likely(v, e, eps) for v, e in (likely_product(d, w.T, sd), likely_product(d.T, x.T, sd.T))]
