"""The log-probabilities, losses and the 4-bit format in 64 bits, one row and one formula at a time, and how far fp32 may be off them."""
import math

import torch

EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # half a step, relative to the value


def rows(logits, T, tokens):
    """logp, entropy [N] and ln p [N, V] in 64 bits; T a number or [N]."""
    x = logits.double()
    T = torch.as_tensor(T, dtype=torch.float64).reshape(-1, 1)
    m = x.max(1, keepdim=True).values
    y = torch.where(torch.isinf(x) & (x < 0), x, (x - m) / T)
    lp = y - y.exp().sum(1, keepdim=True).log()
    H = -torch.where(lp.exp() > 0, lp.exp() * lp, torch.zeros_like(lp)).sum(1)
    ok = (tokens >= 0) & (tokens < x.shape[1])
    t = tokens.long().clamp(0, x.shape[1] - 1)
    logp = torch.where(ok, lp.gather(1, t[:, None]).squeeze(1), math.nan)
    return logp, H, lp


def gradient(lp, H, tokens, T, a, b=None):
    """d/dlogits for upstream gradients a (of logp) and b (of the entropy)."""
    T = torch.as_tensor(T, dtype=torch.float64).reshape(-1, 1)
    p = lp.exp()
    hot = torch.zeros_like(p).scatter_(1, tokens.long().clamp(0, p.shape[1] - 1)[:, None], 1.0)
    g = a.double()[:, None] * (hot - p)
    if b is not None:
        g = g - b.double()[:, None] * torch.where(p > 0, p * (lp + H[:, None]), torch.zeros_like(p))
    return g / T


def spread(lp):
    """The mean distance of a row's logits from its largest, in exponents of 2: what rounds the terms of its sum."""
    d = torch.where(lp.exp() > 0, lp.exp() * (lp.max(1, keepdim=True).values - lp), torch.zeros_like(lp)).sum(1)
    return d / math.log(2)


def logp_bound(lp, value):
    """fp32 error of a log-probability: half a step of the result, and the relative error of the sum of exponentials.  A term's
    exponent t is off by three roundings (c, the difference, the product) of half a step each, the exponential by a step, and a thread
    adds up to V / 256 terms, of which each addition is half a step, 64 lanes' sums another six."""
    V = lp.shape[1]
    return 2.0 ** -24 * (value.abs() + 3 * math.log(2) * (spread(lp) + 60) + 2 + V / 256 + 8 + 6)


def grad_bound(g, lp, H, T, a, b, dtype):
    """Error of a gradient: its rounding, and fp32 errors of e (k0 + k1 t) relative to its two parts."""
    T = torch.as_tensor(T, dtype=torch.float64).reshape(-1, 1)
    t = torch.where(lp.exp() > 0, lp, torch.zeros_like(lp))
    size = lp.exp() * (a.double().abs()[:, None] + (0 if b is None else b.double().abs()[:, None] * (t.abs() + 2 * H[:, None] + 20))) / T
    terms = 3 * (t.abs() + 60) + lp.shape[1] / 256 + 24
    return EPS[dtype] * g.abs() + 2.0 ** -24 * terms * size + 1e-37


def assert_within(got, want, bound, what=""):
    got = got.double().cpu()
    # what lies beyond fp32's range (a masked token's log-probability at a low temperature: -3.4e38 / 0.7) rounds to an infinity there
    want = torch.where(want.abs() > torch.finfo(torch.float32).max, torch.sign(want) * math.inf, want)
    both = torch.isnan(want)
    assert torch.equal(torch.isnan(got), both), (what, "NaN at other places")
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), (what, "infinities")
    off = ((got - want).abs() - bound)[~both & ~inf]
    assert off.numel() == 0 or float(off.max()) <= 0, (what, "over by", float(off.max()), float((got - want)[~both & ~inf].abs().max()))


# ---- 4 bits ----

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def mx4(x):
    """codes [N, K / 2], scales [N, K / 32] and values [N, K] of the rows of x."""
    N, d = x.shape
    K = -(-d // 128) * 128
    v = torch.zeros(N, K, dtype=torch.float64)
    v[:, :d] = x.double()
    v = v.view(N, -1, 32)
    bad = ~torch.isfinite(v).all(2)
    top = torch.where(bad, 1.0, v.abs().nan_to_num(0.0, 0.0).amax(2))
    e = torch.frexp(top).exponent - 1 - 2
    e = torch.where(top > 0, e, torch.full_like(e, -127)).clamp(min=-127)
    s = torch.ldexp(torch.ones((), dtype=torch.float64), e)
    m = (v.nan_to_num(0.0, 0.0, 0.0) / s[..., None]).abs()
    mid = (GRID[:-1] + GRID[1:]) / 2
    code = torch.zeros_like(m, dtype=torch.int64)
    for k in range(7):                                    # ties: to the even code
        code += ((m > mid[k]) | ((m == mid[k]) & (k % 2 == 1))).long()
    sign = torch.signbit(v).long()
    values = torch.where(sign == 1, -GRID[code], GRID[code]) * s[..., None]
    code = code + 8 * sign
    code[bad] = 0
    values[bad] = math.nan
    scale = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    code = code.view(N, K)
    return (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8), scale, values.view(N, K)
