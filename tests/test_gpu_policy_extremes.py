"""The policy loss where a ratio or a KL term leaves fp32's range: far from the old or the reference policy, tokens that are masked, by every
kernel that forms a row's loss."""
import math

import pytest
import torch

import token_loss_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = math.inf
LOWEST = {torch.float32: torch.finfo(torch.float32).min, torch.bfloat16: torch.finfo(torch.bfloat16).min}
MOST = torch.finfo(torch.float32).max


@pytest.fixture(scope="module")
def difr():
    import paper_2511_02620_amd as m
    m.load_library()
    return m


# logp - old, ref - logp, advantage, what the token's own logit becomes
ROWS = [(0.0, 80.0, 1.0, None), (0.0, 100.0, -1.0, None), (0.0, 699.0, 1.0, None), (0.0, 701.0, 1.0, None), (0.0, 1e4, -1.0, None),
        (0.0, 3e38, 1.0, None), (80.0, 0.1, -1.0, None), (100.0, 0.1, -1.0, None), (699.0, 0.1, -1.0, None), (701.0, 0.1, -1.0, None),
        (1e4, 0.1, -2.0, None), (3e38, 0.1, -1.0, None), (1e4, 0.1, 1.0, None), (701.0, -0.1, 0.0, None), (1e4, -0.1, 0.0, None),
        (-1e4, -1e4, 1.0, None), (-1e4, -1e4, -1.0, None), (0.0, -INF, 0.5, None), (0.1, 0.2, -0.5, None),
        ("old", "ref", 1.0, "lowest"), ("old", "ref", -1.0, "lowest"), ("old", "ref", 1.0, -INF), ("old", "ref", -1.0, -INF), ("old", "ref", -1.0, -1e4)]


# rows held in registers by 256 and by 512 threads, with the next row's copies, with LDS, read twice, and shared among workgroups
@pytest.mark.parametrize("N,V,dtype", [(24, 900, torch.float32), (24, 50003, torch.bfloat16), (70, 151936, torch.bfloat16),
                                       (66, 100003, torch.float32), (66, 151936, torch.float32), (24, 100003, torch.bfloat16)])
@pytest.mark.parametrize("eta", [0.0, 0.01])
def test_ratios_and_divergences_beyond_the_range(difr, N, V, dtype, eta):
    g = torch.Generator().manual_seed(V)
    x = (torch.randn(N, V, generator=g) * 2).to(dtype)
    tok = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    A = torch.randn(N, generator=g)
    for n, (_, _, adv, own) in enumerate(ROWS):
        A[n] = adv
        if own is not None:
            x[n, tok[n]] = LOWEST[dtype] if own == "lowest" else own
    logp, H, lp = ref.rows(x, 1.0, tok)
    old, rl = logp.clone(), logp.clone()
    for n, (dr, dk, _, own) in enumerate(ROWS):
        old[n] = -9.0 if own is not None else logp[n] - dr
        rl[n] = -11.0 if own is not None else logp[n] + dk
    old, rl = old.float(), rl.float()
    beta, lo, hi = 0.07, 0.2, 0.3
    dev = lambda t: t.to(DEV)  # noqa: E731
    call = dict(old_logp=dev(old), ref_logp=dev(rl), clip_low=lo, clip_high=hi, kl_coef=beta, entropy_coef=eta)
    got = difr.policy_loss(dev(x), 1.0, dev(tok), dev(A), **call)

    # the definition; e^u is a number, however large, so that an advantage of 0 leaves nothing of it, and e^d outgrows d
    u, d = logp - old.double(), rl.double() - logp
    r = u.exp().clamp(max=1e300)
    Ad = A.double()
    cut = r.clamp(1 - lo, 1 + hi)
    clipped = r * Ad > cut * Ad
    kl = torch.where(d > 700, torch.full_like(d, INF), torch.expm1(d) - d)
    each = torch.where(clipped, -cut * Ad, -r * Ad) + beta * kl - eta * H
    a = torch.where(clipped, torch.zeros_like(r), -r * Ad) - beta * torch.expm1(d)
    lb = ref.logp_bound(lp, logp.clamp(min=-60))
    hb = 3 * eta * ref.logp_bound(lp, lp.min(1).values.clamp(min=-60))
    # a ratio and e^d move by the exponent's error (old and ref are exact inputs), relative to themselves, a function of a 64-bit
    # argument is good to 2e-7 of its value
    rb, kb = r * (lb + 2e-7), (d.exp() + 1) * (lb + 2e-7)
    kb[torch.isinf(kl)] = 0
    e = ref.EPS[torch.float32]
    each_bound = (e * each.abs() + rb * Ad.abs() + beta * kb + hb).nan_to_num(INF)
    for o in (got, difr.policy_loss(dev(x), 1.0, dev(tok), dev(A), want_grad=False, **call)):
        ref.assert_within(o["kl"], kl, (e * kl + kb).nan_to_num(INF), "kl")
        ref.assert_within(o["token_loss"], each, each_bound, "token loss")
        assert o["loss"].item() == INF
        assert torch.equal((o["flags"].cpu() & difr.FLAG_CLIPPED) != 0, clipped)
        assert (o["kl"] >= 0).all()
    # a row is right where its gradient is a number in fp32 throughout; where it is not, no entry of it passes for one that is right
    grad = ref.gradient(lp, H, tok, 1.0, a / N, torch.full((N,), -eta / N) if eta else None)
    slack = ((rb * Ad.abs() + beta * kb) / N).nan_to_num(INF)[:, None]
    lim = ref.grad_bound(grad, lp, H, 1.0, a / N, torch.full((N,), -eta / N) if eta else None, dtype) + slack
    far = a.abs() / N > 1e30
    near = ~far
    ref.assert_within(got["grad"][dev(near)], grad[near], lim[near], "gradient")
    G = got["grad"].cpu().double()
    want = torch.where(grad.abs() > MOST, torch.sign(grad) * INF, grad)
    right = (G - want).abs() <= lim
    live = lp > -80
    assert (right | ~torch.isfinite(G) | ~live)[far].all()
    assert not (torch.isfinite(G) & ~torch.isfinite(want) & live).any() and torch.isfinite(G[[0, 6]]).all()
