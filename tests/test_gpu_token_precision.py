"""How exact the log-probabilities, entropies and gradients are on rows where fp32 has to be handled with care: one token that has nearly all of
the probability, and logits that rise along the vocabulary.

Bounds.  The reference of a row's exponents is its largest logit, whose term is 1 exactly.  Another term's exponent t is off by two
roundings of half a step (difference, product with its rest) and, as the rest of the factor is taken at the vector's largest logit, by two
halves more, the exponential by a step (two halves), its sum with the other terms of a vector by three halves; sums from there on are 64 bits.  A new maximum multiplies what came before it: three halves each time, and four for each of
the orders that it is higher by, which are orders that those terms are below the largest in the end."""
import math

import pytest
import torch

import token_loss_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = 2.0 ** -24
LN2 = math.log(2)


@pytest.fixture(scope="module")
def difr():
    import paper_2511_02620_amd as m
    m.load_library()
    return m


def _peaked(seed, V, dtype, T):
    """Rows of N(0, 3) noise in which the token has all but 1e-1 ... 1e-12 of the probability, at several places."""
    g = torch.Generator().manual_seed(seed)
    rest, at = [1e-1, 1e-3, 1e-5, 1e-7, 1e-9, 1e-12], [0, V // 7, V // 2, V - 4000, V - 1]
    N = len(rest) * len(at)
    x = (torch.randn(N, V, generator=g) * 3).to(dtype)
    tok = torch.tensor([at[n % len(at)] for n in range(N)], dtype=torch.int32)
    others = x.double() / T
    others.scatter_(1, tok.long()[:, None], -math.inf)
    q = torch.tensor([rest[n // len(at)] for n in range(N)]).double()
    x.scatter_(1, tok.long()[:, None], (T * (others.logsumexp(1) + torch.log1p(-q) - q.log())).to(dtype)[:, None])
    return x, tok, g


def _exact(x, T, tok):
    """logp, entropy, ln p and 1 - p of the token in 64 bits, without the cancellation of ln p - max."""
    y = x.double() / T
    m = y.max(1, keepdim=True).values
    t = tok.long()[:, None]
    e = (y - m).exp()
    others = e.scatter(1, t, 0.0).sum(1)
    own = e.gather(1, t).squeeze(1)
    logp = -torch.log1p(others / own)
    lp = y - m - (others + own).log()[:, None]
    lp.scatter_(1, t, logp[:, None])
    H = -(lp.exp() * lp).nan_to_num(0).sum(1)
    return logp, H, lp, others / (others + own)


def _errors(lp, rises):
    """What ln S, and the entropy, may be off by (rises: halves for the new maxima that a wave meets)."""
    p, t = lp.exp(), ((lp - lp.max(1, keepdim=True).values) / LN2).abs()
    t = torch.where(p > 0, t, torch.zeros_like(t))
    rest = p * (t > 0)
    # the largest logit's vector rounds its others away, at most all of them
    ln_s = HALF * ((rest * (4 * LN2 * t + 5)).sum(1) + rest.sum(1) * rises) + torch.minimum(torch.full_like(p[:, 0], 3 * HALF), rest.sum(1))
    return ln_s, ln_s + HALF * LN2 * (rest * t * (4 * LN2 * t + 11 + rises)).sum(1)


# a workgroup a row, 1024 threads a row, and rows that are shared; both losses' own kernels in the test below
@pytest.mark.parametrize("repeat,V", [(1, 9001), (1, 60000), (1, 128256), (3, 128256)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1.0, 0.7, 0.6, 1.3])
def test_tokens_that_stand_out(difr, repeat, V, dtype, T):
    T = float(torch.tensor(T))
    x, tok, g = _peaked(V, V, dtype, T)
    logp, H, lp, gone = _exact(x, T, tok)
    ln_s, ent = _errors(lp, 40)
    N = x.shape[0] * repeat
    a = torch.randn(N, generator=g)
    rep = lambda t: t.repeat(repeat, *[1] * (t.dim() - 1))  # noqa: E731
    xd, td = rep(x).to(DEV), rep(tok).to(DEV)
    o = difr.token_logprob(xd, T, td, want_entropy=True)
    assert (o["logp"] <= 0).all() and (o["entropy"] >= 0).all()
    ref.assert_within(o["logp"], rep(logp), rep(ln_s) + (HALF + 2e-7) * rep(logp).abs())
    ref.assert_within(o["entropy"], rep(H), rep(ent) + (HALF + 2e-7) * rep(H).abs())
    got = difr.token_logprob_backward(xd, T, td, o["stats"], a.to(DEV)).double().cpu()
    own = got.gather(1, rep(tok).long()[:, None]).squeeze(1)
    assert (own * a >= 0).all(), "the sign of the token's gradient"
    # S is kept in fp32 between the two calls; 1 - p moves as ln p does
    ref.assert_within(own, a.double() * rep(gone) / T, (a.abs() / T) * (rep(ln_s) + 2 * HALF) + (ref.EPS[dtype] + 2e-7) * (a * rep(gone)).abs() / T + 1e-37)
    w = torch.full((N,), 1.0)
    for old in (None, rep(logp).float()):
        p = difr.policy_loss(xd, T, td, a.to(DEV), w.to(DEV), old_logp=None if old is None else old.to(DEV), want_entropy=True)
        assert (p["logp"] <= 0).all() and (p["entropy"] >= 0).all()
        ref.assert_within(p["logp"], rep(logp), rep(ln_s) + (HALF + 2e-7) * rep(logp).abs())
        ref.assert_within(p["entropy"], rep(H), rep(ent) + (HALF + 2e-7) * rep(H).abs())
        own = p["grad"].double().cpu().gather(1, rep(tok).long()[:, None]).squeeze(1)
        assert (own * a <= 0).all(), "the sign of the token's gradient"


@pytest.mark.parametrize("N,V", [(8, 20000), (70, 128256), (8, 128256)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_of_tokens_that_stand_out(difr, N, V, dtype):
    """Entries of a row that fall by 1 - p as a whole: each is right relative to itself."""
    T = float(torch.tensor(0.7))
    x, tok, g = _peaked(V + 1, V, dtype, T)
    x, tok = x.repeat(3, 1)[:N], tok.repeat(3)[:N]
    logp, H, lp, gone = _exact(x, T, tok)
    a = torch.randn(N, generator=g)
    ln_s, _ = _errors(lp, 40)
    want = ref.gradient(lp, H, tok, T, a)
    want.scatter_(1, tok.long()[:, None], (a * gone / T)[:, None])
    t = (lp - lp.max(1, keepdim=True).values).abs().clamp(max=200)
    # the exponent's factor is rounded, not its rest, where the gradient is bf16; coefficients of the backward call in fp32, six roundings
    lim = want.abs() * (ref.EPS[dtype] + HALF * (4 * t + 2 * t + 8) + (ln_s + 2 * HALF)[:, None])
    lim.scatter_(1, tok.long()[:, None], ((a.abs() / T) * (ln_s + 2 * HALF) + (ref.EPS[dtype] + 2e-7) * (a * gone).abs() / T)[:, None])
    xd, td = x.to(DEV), tok.to(DEV)
    o = difr.token_logprob(xd, T, td)
    ref.assert_within(difr.token_logprob_backward(xd, T, td, o["stats"], a.to(DEV)), want, lim + 1e-37, "backward")
    p = difr.policy_loss(xd, T, td, -a.to(DEV), torch.ones(N, device=DEV))
    ref.assert_within(p["grad"], want, lim + 1e-37, "policy")


@pytest.mark.parametrize("N,V", [(6, 9001), (6, 128256), (70, 128256)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_rise_and_fall(difr, N, V, dtype):
    """Logits that rise along the vocabulary by 3, 30 and 300, in steps and evenly, and that fall: every vector may be a new maximum."""
    g = torch.Generator().manual_seed(V)
    ramp = torch.arange(V) / V
    x = torch.randn(N, V, generator=g) * 0.5
    for n in range(N):
        x[n] += [3, 30, 300, 30, -30, 0][n % 6] * (ramp if n % 6 != 3 else (ramp * 20).floor() / 20)
    x = x.to(dtype)
    tok = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    tok[::2] = x[::2].argmax(1).int()
    logp, H, lp, _ = _exact(x, 1.0, tok)
    # a wave may meet a new maximum in each of its vectors, 512 or 256 entries apart, four waves and more to a row
    rounds = V / (2048 if dtype == torch.bfloat16 else 1024)
    ln_s, ent = _errors(lp, 3 * rounds + 9)
    o = difr.token_logprob(x.to(DEV), 1.0, tok.to(DEV), want_entropy=True)
    p = difr.policy_loss(x.to(DEV), 1.0, tok.to(DEV), torch.ones(N, device=DEV), want_entropy=True)
    for r in (o, p):
        assert (r["logp"] <= 0).all() and (r["entropy"] >= 0).all()
        ref.assert_within(r["logp"], logp, ln_s + (HALF + 2e-7) * logp.abs())
        ref.assert_within(r["entropy"], H, ent + (HALF + 2e-7) * H.abs())


@pytest.mark.parametrize("N,V", [(5, 777), (5, 100003), (70, 40000)])
@pytest.mark.parametrize("T", [1e-45, 1e-39, 1e-38, 1e38, 3.4e38])
def test_temperatures_at_the_ends_of_the_range(difr, N, V, T):
    """A temperature that is positive and finite has a log-probability, be it 0 or far beyond fp32's range, or -ln V."""
    g = torch.Generator().manual_seed(N)
    x = torch.randn(N, V, generator=g)
    tok = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    tok[0] = x[0].argmax()
    T = float(torch.tensor(T))
    y = x.double() / T
    logp = y.gather(1, tok.long()[:, None]).squeeze(1) - y.logsumexp(1)
    for kw in (dict(), dict(temperatures=torch.full((N,), T, device=DEV))):
        o = difr.token_logprob(x.to(DEV), T, tok.to(DEV), want_entropy=True, **kw)
        assert o["flags"].eq(0).all()
        # exponents of 1e-38 and less leave every term 1, of 1e38 and more none but the largest
        ref.assert_within(o["logp"], logp, (HALF + 2e-7) * logp.abs())
        assert (o["entropy"] - (math.log(V) if T > 1 else 0.0)).abs().max() < 3e-7 * math.log(V)
