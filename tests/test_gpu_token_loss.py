"""Log-probabilities of logged tokens, the clipped policy loss and the preference loss against their definitions in 64 bits, and their
gradients against formulas and differences."""
import math

import pytest
import torch

import token_loss_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LOWEST = {torch.float32: torch.finfo(torch.float32).min, torch.bfloat16: torch.finfo(torch.bfloat16).min}
INF = math.inf


@pytest.fixture(scope="module")
def difr():
    import paper_2511_02620_amd as m
    m.load_library()
    return m


def _logits(seed, N, V, dtype, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(N, V, generator=g) * scale).to(dtype), torch.randint(0, V, (N,), generator=g, dtype=torch.int32), g


def _on_device(x, offset=0, gap=0):
    """x [N, V] on the GPU with `gap` elements between its rows, `offset` elements into an allocation."""
    N, V = x.shape
    buf = torch.full((offset + N * (V + gap) + 8,), 7.0, dtype=x.dtype, device=DEV)
    view = buf[offset:offset + N * (V + gap)].view(N, V + gap)[:, :V]
    view.copy_(x)
    return view


SHAPES = [(1, 1), (3, 2), (2, 7), (4, 8), (5, 9), (3, 255), (4, 1000), (6, 1024), (3, 2049), (2, 8197), (3, 40001), (2, 151936), (700, 130),
          (20, 100003), (64, 98304), (65, 98304)]


@pytest.mark.parametrize("N,V", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset,gap", [(0, 0), (1, 0), (3, 5)])
def test_forward_and_backward(difr, N, V, dtype, offset, gap):
    x, tok, g = _logits(N * 1000 + V, N, V, dtype)
    T = torch.rand(N, generator=g) + 0.5
    a, b = torch.randn(N, generator=g), torch.randn(N, generator=g)
    xd, td, Td = _on_device(x, offset, gap), tok.to(DEV), T.to(DEV)
    logp, H, lp = ref.rows(x, T, tok)
    o = difr.token_logprob(xd, 1.0, td, temperatures=Td, want_entropy=True)
    ref.assert_within(o["logp"], logp, ref.logp_bound(lp, logp), "logp")
    # the entropy's two parts, ln S and the mean exponent, have the log-probability's errors
    ref.assert_within(o["entropy"], H, 3 * ref.logp_bound(lp, lp.min(1).values.clamp(min=-60)), "entropy")
    assert o["flags"].eq(0).all()
    plain = difr.token_logprob(xd, 1.0, td, temperatures=Td)
    assert "entropy" not in plain and torch.equal(plain["logp"], o["logp"]) and torch.equal(plain["stats"], o["stats"])
    for up in (b, None):
        want = ref.gradient(lp, H, tok, T, a, up)
        kw = dict(entropy=o["entropy"], grad_entropy=up.to(DEV)) if up is not None else {}
        got = difr.token_logprob_backward(xd, 1.0, td, o["stats"], a.to(DEV), temperatures=Td, **kw)
        assert got.dtype == dtype
        ref.assert_within(got, want, ref.grad_bound(want, lp, H, T, a, up, dtype), "gradient")
        into = _on_device(torch.zeros_like(x), 2, 3)
        assert difr.token_logprob_backward(xd, 1.0, td, o["stats"], a.to(DEV), temperatures=Td, out=into, **kw).data_ptr() == into.data_ptr()
        assert torch.equal(into, got) and into._base.eq(7.0).sum() >= 2 + 3 * N + 8, "entries between the rows"
        same = _on_device(x, offset, gap)
        difr.token_logprob_backward(same, 1.0, td, o["stats"], a.to(DEV), temperatures=Td, out=same, **kw)
        assert torch.equal(same, got), "in place"


@pytest.mark.parametrize("V", [17, 1024, 3001, 9000, 100003])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masks_and_infinities(difr, V, dtype):
    x, tok, g = _logits(V, 12, V, dtype)
    last = V - 1
    x[0, :last] = -INF                               # one entry left
    x[1, :] = -INF                                   # none
    x[2, :] = LOWEST[dtype]                          # nothing but the lowest value: uniform
    x[3, :last] = LOWEST[dtype]
    x[4, V // 2] = math.nan
    x[5, V // 3] = INF
    x[6, 5] = -INF                                   # the token's own entry is masked
    x[7, :] = -1e4
    x[7, last] = 1e4                                 # the largest comes last, far above the others
    x[8, : V // 2] = -INF
    x[9, ::2] = LOWEST[dtype]
    x[10, last - 1] = -INF if V > 1 else 0
    tok[0], tok[3], tok[6], tok[7] = last, last, 5, last
    tok[10], tok[11] = -1, V
    T = 0.7
    Tq = float(torch.tensor(T))
    a, b = torch.randn(12, generator=g), torch.randn(12, generator=g)
    logp, H, lp = ref.rows(x, Tq, tok)
    xd = x.to(DEV)
    o = difr.token_logprob(xd, T, tok.to(DEV), want_entropy=True)
    bad = torch.tensor([1, 4, 5])
    flags = torch.zeros(12, dtype=torch.uint8)
    flags[bad] = difr.FLAG_NONFINITE
    flags[10:] = difr.FLAG_INVALID_CLAIM
    assert torch.equal(o["flags"].cpu(), flags)
    logp[bad], H[bad], lp[bad] = math.nan, math.nan, 0.0
    bound = ref.logp_bound(lp, logp.nan_to_num(0, 0, 0))
    ref.assert_within(o["logp"], logp, bound, "logp")
    ref.assert_within(o["entropy"], H, 3 * bound, "entropy")
    got = difr.token_logprob_backward(xd, T, tok.to(DEV), o["stats"], a.to(DEV), entropy=o["entropy"], grad_entropy=b.to(DEV))
    want = ref.gradient(lp, H.nan_to_num(0), tok, Tq, a, b)
    lim = ref.grad_bound(want, lp, H.nan_to_num(0), Tq, a, b, dtype)
    want[bad] = math.nan
    want[10:] = math.nan
    ref.assert_within(got, want, lim, "gradient")
    # rows without an upstream gradient are zero whatever they hold
    a[bad] = b[bad] = 0.0
    a[10:], b[10] = 0.0, 0.0
    got = difr.token_logprob_backward(xd, T, tok.to(DEV), o["stats"], a.to(DEV), entropy=o["entropy"], grad_entropy=b.to(DEV))
    assert got[[1, 4, 5, 10]].eq(0).all() and torch.isfinite(got[11]).all() == torch.isfinite(o["entropy"][11])


@pytest.mark.parametrize("V", [777, 100003])
def test_bad_temperatures_touch_their_rows_only(difr, V):
    x, tok, _ = _logits(5, 5, V, torch.bfloat16)
    T = torch.tensor([1.0, 0.0, -1.0, math.nan, 2.0])
    o = difr.token_logprob(x.to(DEV), 1.0, tok.to(DEV), temperatures=T.to(DEV), want_entropy=True)
    assert torch.isnan(o["logp"]).tolist() == [False, True, True, True, False]
    assert o["flags"].tolist() == [0, 4, 4, 4, 0]
    got = difr.token_logprob_backward(x.to(DEV), 1.0, tok.to(DEV), o["stats"], torch.ones(5, device=DEV), temperatures=T.to(DEV))
    assert torch.isnan(got).all(1).tolist() == [False, True, True, True, False]


def test_low_and_high_temperatures(difr):
    for T in (1e-3, 0.02, 50.0, 1e6):
        for dtype in (torch.bfloat16, torch.float32):
            x, tok, g = _logits(9, 4, 5000, dtype)
            tok[0] = int(x[0].argmax())
            Tq = float(torch.tensor(T))
            logp, H, lp = ref.rows(x, Tq, tok)
            o = difr.token_logprob(x.to(DEV), T, tok.to(DEV), want_entropy=True)
            # the exponent of an entry is off relative to itself, whatever the temperature made of it
            ref.assert_within(o["logp"], logp, ref.logp_bound(lp, 4 * logp), "logp")
            a = torch.ones(4)
            got = difr.token_logprob_backward(x.to(DEV), T, tok.to(DEV), o["stats"], a.to(DEV))
            want = ref.gradient(lp, H, tok, Tq, a)
            ref.assert_within(got, want, ref.grad_bound(want, lp, H, Tq, a, None, dtype), "gradient")


def test_rows_whose_parts_have_nothing_in_common(difr):
    """Stretches of a long row that different workgroups sum, far apart in scale, without mass, or with a NaN in one entry of one."""
    N, V = 9, 131072
    for dtype in (torch.bfloat16, torch.float32):
        x, tok, g = _logits(31, N, V, dtype)
        ramp = torch.arange(V) // 4096
        x[0] = (x[0].float() + 40.0 * ramp).to(dtype)          # each stretch far above the one before
        x[1] = (x[1].float() - 40.0 * ramp).to(dtype)
        x[2, : V - 3] = -INF
        x[3, 5:] = LOWEST[dtype]
        x[4, ::4096] = -INF
        x[5, 70000] = math.nan
        x[6, V - 1] = INF
        x[7, 60000:61000] = math.nan
        x[8, 4096:8192] = LOWEST[dtype]
        tok[0], tok[2], tok[3] = V - 1, V - 2, 3
        bad = torch.tensor([5, 6, 7])
        logp, H, lp = ref.rows(x, 1.0, tok)
        logp[bad], H[bad], lp[bad] = math.nan, math.nan, 0.0
        o = difr.token_logprob(x.to(DEV), 1.0, tok.to(DEV), want_entropy=True)
        assert [n for n in range(N) if o["flags"][n]] == bad.tolist()
        ref.assert_within(o["logp"], logp, ref.logp_bound(lp, logp.nan_to_num(0, 0, 0)), "logp")
        ref.assert_within(o["entropy"], H, 3 * ref.logp_bound(lp, lp.min(1).values.clamp(min=-60)), "entropy")
        A = torch.randn(N, generator=g)
        got = difr.policy_loss(x.to(DEV), 1.0, tok.to(DEV), A.to(DEV))["grad"]
        want = ref.gradient(lp, H.nan_to_num(0), tok, 1.0, -A.double() / N)
        lim = ref.grad_bound(want, lp, H.nan_to_num(0), 1.0, -A / N, None, dtype)
        want[bad] = math.nan
        ref.assert_within(got, want, lim, "gradient")


def test_no_rows(difr):
    x, t, f = torch.zeros(0, 9, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV), torch.zeros(0, device=DEV)
    assert difr.token_logprob(x, 1.0, t, want_entropy=True)["logp"].shape == (0,)
    assert difr.token_logprob_backward(x, 1.0, t, torch.zeros(0, 2, device=DEV), f).shape == (0, 9)
    o = difr.policy_loss(x, 1.0, t, f)
    assert o["loss"].tolist() == [0.0] and o["grad"].shape == (0, 9)
    off = torch.zeros(1, dtype=torch.int64, device=DEV)
    assert difr.preference_loss(x, 1.0, t, off, 0.1)["loss"].tolist() == [0.0]
    o = difr.preference_loss(x, 1.0, t, torch.zeros(3, dtype=torch.int64, device=DEV), 0.1)   # a pair of empty replies
    assert o["seq_logp"].tolist() == [0.0, 0.0] and abs(o["loss"].item() - math.log(2)) < 1e-7


# ---- policy loss ----

def _policy_ref(x, T, tok, A, w, old, refl, lo, hi, beta, eta):
    logp, H, lp = ref.rows(x, T, tok)
    N = x.shape[0]
    w = torch.full((N,), 1.0 / N, dtype=torch.float64) if w is None else w.double()
    A = A.double()
    r = torch.ones_like(A) if old is None else (logp - old.double()).exp()
    cut = r.clamp(1 - lo, 1 + hi)
    clipped = r * A > cut * A
    each = torch.where(clipped, -cut * A, -r * A)
    a = torch.where(clipped, torch.zeros_like(A), -r * A)
    kl = None
    if refl is not None:
        d = refl.double() - logp
        kl = torch.expm1(d) - d
        each, a = each + beta * kl, a - beta * torch.expm1(d)
    each = each - eta * H
    live = w != 0
    zero = torch.zeros_like(w)
    return dict(loss=(w * each)[live].sum().reshape(1), token_loss=torch.where(live, each, zero), logp=torch.where(live, logp, zero),
                entropy=torch.where(live, H, zero), kl=None if kl is None else torch.where(live, kl, zero),
                clipped=clipped & live, a=torch.where(live, w * a, zero), b=-eta * w, lp=lp, H=H)


# (rows of a workgroup's registers in all their lengths, from one vector to a compute unit's; with LDS; longer ones)
@pytest.mark.parametrize("N,V", [(1, 1), (2, 50), (33, 1024), (5, 8197), (3, 40001), (2, 151936), (300, 515), (259, 20003), (3, 75000),
                                 (3, 100001), (2, 165000), (2, 230001), (66, 100001), (66, 151936), (64, 98304)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("old,refl,weights,eta", [(1, 1, 1, 0.0), (1, 1, 1, 0.02), (0, 0, 0, 0.0), (1, 0, 1, 0.01), (0, 1, 0, 0.0)])
def test_policy_loss(difr, N, V, dtype, old, refl, weights, eta):
    x, tok, g = _logits(N + V, N, V, dtype, 2.0)
    T = torch.rand(N, generator=g) + 0.6
    logp, _, _ = ref.rows(x, T, tok)
    A = torch.randn(N, generator=g)
    w = torch.rand(N, generator=g) * (torch.rand(N, generator=g) > 0.3) if weights else None
    o_l = (logp + 0.3 * torch.randn(N, generator=g)).float() if old else None
    r_l = (logp + 0.5 * torch.randn(N, generator=g)).float() if refl else None
    beta = 0.07 if refl else 0.0
    if w is not None and N > 2:
        x[1], w[1] = math.nan, 0.0                    # what is left out may hold anything
        tok[1] = -100
    want = _policy_ref(x, T, tok, A, w, o_l, r_l, 0.2, 0.3, beta, eta)
    if w is not None and N > 2:
        want["lp"][1], want["H"][1] = 0.0, 0.0
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    xd = _on_device(x, 1, 2)
    call = dict(weights=dev(w), old_logp=dev(o_l), ref_logp=dev(r_l), clip_low=0.2, clip_high=0.3, kl_coef=beta, entropy_coef=eta,
                temperatures=dev(T))
    got = difr.policy_loss(xd, 1.0, dev(tok), dev(A), want_entropy=True, **call)
    lb = ref.logp_bound(want["lp"], want["logp"])
    ref.assert_within(got["logp"], want["logp"], lb)
    ref.assert_within(got["entropy"], want["entropy"], 3 * ref.logp_bound(want["lp"], want["lp"].min(1).values.clamp(min=-60)))
    # a ratio moves by its log-probability's error, relative to itself
    r = torch.ones(N, dtype=torch.float64) if o_l is None else (want["logp"] - o_l.double()).exp()
    e = ref.EPS[torch.float32]
    each_bound = e * want["token_loss"].abs() + lb * (r * A.abs() + beta * ((r_l.double() - want["logp"]).exp() + 1) if refl else r * A.abs())
    each_bound += 3 * eta * ref.logp_bound(want["lp"], want["lp"].min(1).values.clamp(min=-60))
    dead = want["token_loss"] == 0
    each_bound[dead & (torch.zeros(N) if w is None else w).eq(0) & torch.tensor(weights == 1)] = 0
    ref.assert_within(got["token_loss"], want["token_loss"], each_bound)
    wt = torch.full((N,), 1.0 / N) if w is None else w
    total = float((wt.double().abs() * each_bound).nan_to_num(0).sum())
    ref.assert_within(got["loss"], want["loss"], total + e * want["loss"].abs() + 1e-37)
    if refl:
        ref.assert_within(got["kl"], want["kl"], e * want["kl"] + lb * ((r_l.double() - want["logp"]).exp() + 1) * (want["kl"] != 0))
    assert torch.equal((got["flags"].cpu() & difr.FLAG_CLIPPED) != 0, want["clipped"])
    grad = ref.gradient(want["lp"], want["H"], tok, T, want["a"], want["b"] if eta else None)
    if w is not None:
        grad[w == 0] = 0.0
    slack = (wt.double() * lb * (r * A.abs() + (beta * (r_l.double() - want["logp"]).exp() if refl else 0))).nan_to_num(0)[:, None] / T[:, None]
    lim = ref.grad_bound(grad, want["lp"], want["H"], T, want["a"], want["b"] if eta else None, dtype) + slack
    ref.assert_within(got["grad"], grad, lim, "gradient")
    # without the gradient the row is summed in another order: two sums of the same bound
    again = difr.policy_loss(xd, 1.0, dev(tok), dev(A), want_entropy=True, want_grad=False, **call)
    assert "grad" not in again and torch.equal(again["flags"], got["flags"])
    ref.assert_within(again["logp"], want["logp"], lb)
    ref.assert_within(again["token_loss"], want["token_loss"], each_bound)
    ref.assert_within(again["loss"], want["loss"], total + e * want["loss"].abs() + 1e-37)
    if torch.isnan(x).any() or V > 160000:
        return
    same = _on_device(x, 1, 2)
    o = difr.policy_loss(same, 1.0, dev(tok), dev(A), out=same, **call)
    assert o["grad"].data_ptr() == same.data_ptr() and torch.equal(same, got["grad"]), "in place"


@pytest.mark.parametrize("V", [50000, 80003, 128256, 151936])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_policy_rows_that_follow_each_other(difr, V, dtype):
    """Rows that a workgroup takes one after another are those of smaller batches, to the bit, whatever lies between them.  (A batch of
    256 rows or fewer gives a row of under 39 vectors of 16 bytes to each of 256 threads more threads, which sum it in another order.)"""
    N = 700
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn(N, V + 3, generator=g, device=DEV).mul_(2).to(dtype)[:, :V]
    tok = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    A, u = torch.randn(N, generator=g, device=DEV), torch.rand(N, generator=g, device=DEV)
    w = torch.where(u < 0.3, torch.zeros_like(u), u)
    x[u < 0.1], w[256:259] = math.nan, 0.0
    old = torch.full((N,), -11.0, device=DEV)

    def call(rows, **kw):
        return difr.policy_loss(x[rows], 1.0, tok[rows], A[rows], w[rows], old_logp=old[rows], ref_logp=old[rows], kl_coef=0.1, **kw)

    got = call(slice(0, N))
    assert got["grad"][w == 0].eq(0).all() and torch.isfinite(got["grad"]).all()
    step = 175 if V * x.element_size() >= 39 * 256 * 16 else 350
    for first in range(0, N, step):
        rows = slice(first, first + step)
        part = call(rows)
        for k in ("token_loss", "logp", "kl", "flags", "grad"):
            assert torch.equal(part[k], got[k][rows]), (first, k)
    del part
    again = call(slice(0, N), out=x)
    assert torch.equal(again["grad"], got["grad"]), "in place"


@pytest.mark.parametrize("V", [900, 50000, 100003])
def test_policy_rows_that_cannot_be_scored_are_loud(difr, V):
    x, tok, g = _logits(3, 6, V, torch.bfloat16)
    x[1, 5], tok[2], x[3, :] = math.nan, V, -INF
    A, w = torch.ones(6, device=DEV), torch.full((6,), 0.1, device=DEV)
    o = difr.policy_loss(x.to(DEV), 1.0, tok.to(DEV), A, w, want_entropy=True)
    assert torch.isnan(o["token_loss"]).tolist() == [False, True, True, True, False, False]
    assert torch.isnan(o["loss"]).item()
    assert torch.isnan(o["grad"]).all(1).tolist() == [False, True, True, True, False, False]
    w[1:4] = 0.0
    o = difr.policy_loss(x.to(DEV), 1.0, tok.to(DEV), A, w)
    assert torch.isfinite(o["loss"]).item() and o["grad"][1:4].eq(0).all() and o["flags"].tolist() == [0] * 6


def test_policy_clip_sides(difr):
    """Ratios on both sides of the clip with both signs of the advantage, infinite bounds among them."""
    x = torch.zeros(8, 4)
    tok = torch.zeros(8, dtype=torch.int32)
    old = math.log(0.25) - torch.tensor([0.5, 0.5, -0.5, -0.5, 0.05, 0.05, -0.05, -0.05])    # ratios e^.5, e^-.5, e^+-.05
    A = torch.tensor([1.0, -1.0] * 4)
    o = difr.policy_loss(x.to(DEV), 1.0, tok.to(DEV), A.to(DEV), old_logp=old.to(DEV))
    assert (o["flags"] == difr.FLAG_CLIPPED).tolist() == [True, False, False, True, False, False, False, False]
    assert o["grad"].ne(0).any(1).tolist() == [False, True, True, False, True, True, True, True]
    o = difr.policy_loss(x.to(DEV), 1.0, tok.to(DEV), A.to(DEV), old_logp=old.to(DEV), clip_low=1.0, clip_high=INF)
    assert o["flags"].eq(0).all()


# ---- preference loss ----

def _pairs_ref(x, T, tok, off, beta, mask, refs, pw, eps, margin, average):
    logp, H, lp = ref.rows(x, T, tok)
    N, S = x.shape[0], len(off) - 1
    keep = torch.ones(N, dtype=torch.bool) if mask is None else mask != 0
    each = torch.where(keep, logp, torch.zeros_like(logp))
    total, share = torch.zeros(S, dtype=torch.float64), torch.ones(S, dtype=torch.float64)
    for s in range(S):
        n = int(keep[off[s]:off[s + 1]].sum())
        if average and n:
            share[s] = 1.0 / n
        total[s] = each[off[s]:off[s + 1]].sum() * share[s]
    ratio = total - (0 if refs is None else refs.double())
    h = beta * (ratio[0::2] - ratio[1::2]) - margin
    ls = torch.nn.functional.logsigmoid
    loss = -(1 - eps) * ls(h) - eps * ls(-h)
    w = torch.full((S // 2,), 2.0 / S, dtype=torch.float64) if pw is None else pw.double()
    dh = w * beta * (eps * torch.sigmoid(h) - (1 - eps) * torch.sigmoid(-h))
    a = torch.zeros(N, dtype=torch.float64)
    for s in range(S):
        a[off[s]:off[s + 1]] = dh[s // 2] * (1 if s % 2 == 0 else -1) * share[s]
    a = torch.where(keep, a, torch.zeros_like(a))
    return dict(logp=each, seq_logp=total, pair_loss=loss, loss=(w * loss).sum().reshape(1), a=a, lp=lp, H=H, h=h, share=share, w=w)


@pytest.mark.parametrize("off,N", [([0, 3, 7], 7), ([2, 2, 9, 9, 20], 24), ([0, 300, 301, 301, 640, 700, 900], 900), ([0, 1, 2], 2)])
@pytest.mark.parametrize("V", [7, 1024, 20011, 100003])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("masked,refs,weights,eps,margin,average", [(1, 1, 1, 0.1, 0.5, 0), (0, 0, 0, 0.0, 0.0, 0), (1, 1, 0, 1.0, 0.0, 1),
                                                                    (1, 0, 1, 0.0, 1.0, 1)])
def test_preference_loss(difr, off, N, V, dtype, masked, refs, weights, eps, margin, average):
    if N > 100 and V > 10000:
        pytest.skip("the same rows as the smaller ones, at length")
    x, tok, g = _logits(N * V, N, V, dtype, 2.0)
    S, beta, T = len(off) - 1, 0.3, 0.9
    Tq = float(torch.tensor(T))
    mask = (torch.rand(N, generator=g) > 0.4).to(torch.uint8) * 3 if masked else None
    if masked:
        mask[off[-2]:off[-1]] = 0                     # the last reply is masked whole
        x[off[-2]], tok[off[-2]] = math.nan, -100
    logp, _, _ = ref.rows(x, Tq, tok)
    r = torch.randn(S, generator=g) * 2 if refs else None
    pw = torch.rand(S // 2, generator=g) if weights else None
    want = _pairs_ref(x, Tq, tok, off, beta, mask, r, pw, eps, margin, average)
    dead = torch.zeros(N, dtype=torch.bool) if mask is None else mask == 0
    want["lp"][dead], want["H"][dead] = 0.0, 0.0
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    xd = _on_device(x, 1, 1)
    offd = torch.tensor(off, dtype=torch.int64, device=DEV)
    call = dict(mask=dev(mask), ref_seq_logp=dev(r), pair_weights=dev(pw), label_smoothing=eps, margin=margin, average=bool(average))
    got = difr.preference_loss(xd, T, dev(tok), offd, beta, **call)
    lb = torch.where(dead, torch.zeros(()), ref.logp_bound(want["lp"], want["logp"]))
    ref.assert_within(got["logp"], want["logp"], lb)
    e = ref.EPS[torch.float32]
    # every logp is rounded to fp32 and may be off by its bound; a pair's h by the two sums' errors, its loss by no more than that
    sb = torch.stack([lb[off[s]:off[s + 1]].sum() * want["share"][s] for s in range(S)])
    ref.assert_within(got["seq_logp"], want["seq_logp"], sb + e * want["seq_logp"].abs())
    hb = beta * (sb[0::2] + sb[1::2])
    ref.assert_within(got["pair_loss"], want["pair_loss"], hb + e * want["pair_loss"])
    ref.assert_within(got["loss"], want["loss"], (want["w"] * (hb + e * want["pair_loss"])).sum() + e * want["loss"])
    slope = torch.zeros(N, dtype=torch.float64)
    for s in range(S):
        slope[off[s]:off[s + 1]] = want["w"][s // 2] * beta * hb[s // 2] / 4 * want["share"][s]     # sigma' <= 1 / 4
    slope[dead] = 0
    ref.assert_within(got["grad_logp"], want["a"], slope + e * want["a"].abs())
    grad = ref.gradient(want["lp"], want["H"], tok, Tq, want["a"])
    grad[dead] = 0.0
    ref.assert_within(got["grad"], grad, ref.grad_bound(grad, want["lp"], want["H"], Tq, want["a"], None, dtype) + 2 * slope[:, None] / Tq, "gradient")
    outside = [n for n in range(N) if n < off[0] or n >= off[-1]]
    assert got["grad"][outside].eq(0).all()
    again = difr.preference_loss(xd, T, dev(tok), offd, beta, want_grad=False, **call)
    assert "grad" not in again and all(torch.equal(again[k], got[k]) for k in again)
    if masked:
        return
    same = _on_device(x, 1, 1)
    o = difr.preference_loss(same, T, dev(tok), offd, beta, out=same, **call)
    assert torch.equal(same, got["grad"]) and torch.equal(o["logp"], got["logp"]), "in place"


def test_preference_far_from_balance(difr):
    """Log ratios of thousands: the loss is linear on one side and 0 on the other, and so is what flows back."""
    x, tok, g = _logits(2, 8, 64, torch.float32)
    off = torch.tensor([0, 2, 4, 6, 8], dtype=torch.int64, device=DEV)
    r = torch.tensor([-4000.0, 4000.0, 4000.0, -4000.0])
    want = _pairs_ref(x, 1.0, tok, [0, 2, 4, 6, 8], 1.0, None, r, None, 0.0, 0.0, False)
    got = difr.preference_loss(x.to(DEV), 1.0, tok.to(DEV), off, 1.0, ref_seq_logp=r.to(DEV))
    assert got["pair_loss"][0].item() == 0.0 and got["grad"][:4].eq(0).all()
    ref.assert_within(got["pair_loss"], want["pair_loss"], 2e-7 * want["pair_loss"] + 1e-5)
    ref.assert_within(got["grad_logp"], want["a"], 2.0 ** -24 * want["a"].abs() + 1e-37)


# ---- gradients against differences ----

def test_gradients_are_the_slopes(difr):
    """Central differences of the losses along random directions.  A loss is a sum of fp32 log-probabilities of about 5 with errors of
    some 1e-6 each, over N of them with weights 1 / N: a difference over 2 h = 0.04 is good to 1e-6 / 0.04 = 3e-5, and the third
    derivative (below 1 per unit direction, spread over the vocabulary) adds h^2 / 6 = 7e-5."""
    N, V, h = 24, 40, 0.02
    x, tok, g = _logits(4, N, V, torch.float32, 1.5)
    logp = ref.rows(x, 1.0, tok)[0]
    A, w = torch.randn(N, generator=g), torch.full((N,), 1.0 / N)
    # ratios well inside or outside the clip, so that no difference crosses its edge
    old = (logp - torch.tensor([0.0, 0.6, -0.6] * 8)).float()
    rl = (logp + 0.3 * torch.randn(N, generator=g)).float()
    off = torch.tensor([0, 5, 11, 17, 24], dtype=torch.int64, device=DEV)
    d = lambda t: t.to(DEV)  # noqa: E731

    def policy(z):
        return difr.policy_loss(d(z), 1.0, d(tok), d(A), d(w), old_logp=d(old), ref_logp=d(rl), kl_coef=0.5, entropy_coef=0.3)

    def pairs(z):
        return difr.preference_loss(d(z), 1.0, d(tok), off, 0.2, average=True, label_smoothing=0.05)

    for f in (policy, pairs):
        grad = f(x)["grad"].double().cpu()
        for k in range(6):
            u = torch.randn(N, V, generator=g)
            u /= u.norm(dim=1, keepdim=True)
            slope = (f(x + h * u)["loss"].item() - f(x - h * u)["loss"].item()) / (2 * h)
            assert abs(slope - float((grad * u.double()).sum())) < 4e-4, (f.__name__, k)


# ---- streams, graphs ----

@pytest.mark.parametrize("V", [30011, 100003])
def test_other_streams_and_repeats(difr, V):
    x, tok, g = _logits(8, 40, V, torch.bfloat16)
    xd, td, A = x.to(DEV), tok.to(DEV), torch.randn(40, generator=g).to(DEV)
    first = difr.policy_loss(xd, 1.0, td, A, want_entropy=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = difr.policy_loss(xd, 1.0, td, A, want_entropy=True)
    side.synchronize()
    for k in first:
        assert torch.equal(first[k], other[k]), k


@pytest.mark.parametrize("V", [5003, 100003])
def test_a_step_is_captured_and_replayed(difr, V):
    N = 48
    off = torch.tensor([0, 10, 24, 30, 48], dtype=torch.int64, device=DEV)
    xd, td = torch.zeros(N, V, dtype=torch.bfloat16, device=DEV), torch.zeros(N, dtype=torch.int32, device=DEV)
    A, w = torch.zeros(N, device=DEV), torch.zeros(N, device=DEV)

    def load(seed):
        x, tok, g = _logits(seed, N, V, torch.bfloat16)
        xd.copy_(x), td.copy_(tok), A.copy_(torch.randn(N, generator=g)), w.copy_((torch.rand(N, generator=g) > 0.3).float() / N)

    def step():
        o = difr.token_logprob(xd, 0.8, td, want_entropy=True)
        p = difr.policy_loss(xd, 0.8, td, A, w, old_logp=o["logp"], ref_logp=o["logp"], kl_coef=0.1, entropy_coef=0.01)
        q = difr.preference_loss(xd, 0.8, td, off, 0.2)
        b = difr.token_logprob_backward(xd, 0.8, td, o["stats"], A, entropy=o["entropy"], grad_entropy=w)
        return [*o.values(), *p.values(), *q.values(), b]

    load(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in (21, 22, 23, 24):
        load(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        eager = step()
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(got, eager)):
            assert torch.equal(x, y), (seed, i)


def test_more_rows_than_a_grid_of_threads_counts(difr):
    N, V = (1 << 24) + 5, 3
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(N, V, generator=g, device=DEV)
    tok = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    lp = torch.log_softmax(x.double(), 1)
    want = lp.gather(1, tok.long()[:, None]).squeeze(1)
    # three exponents, their sum, its logarithm and the result: some 10 roundings of numbers below 12
    bound = 10 * 2.0 ** -24 * 12
    o = difr.token_logprob(x, 1.0, tok, want_entropy=True)
    assert (o["logp"] - want).abs().max() < bound and o["flags"].eq(0).all()
    assert (o["entropy"] + (lp.exp() * lp).sum(1)).abs().max() < bound
    A = torch.randn(N, generator=g, device=DEV)
    for kw in (dict(want_grad=False), dict(out=x)):
        p = difr.policy_loss(x, 1.0, tok, A, **kw)
        assert (p["logp"] - want).abs().max() < bound and torch.equal(p["token_loss"], -A)
    empty = torch.zeros(2 * N + 1, dtype=torch.int64, device=DEV)                   # as many pairs of empty replies
    q = difr.preference_loss(x[:1], 1.0, tok[:1], empty, 0.1, want_grad=False)
    assert q["pair_loss"].shape[0] == N and (q["pair_loss"] - math.log(2)).abs().max() < 1e-7
    back = -(A.double() / N)[:, None] * (torch.nn.functional.one_hot(tok.long(), V) - lp.exp())
    assert ((x - back).abs() <= 2 * bound * (A.double().abs() / N)[:, None]).all()


def test_a_vocabulary_beyond_the_columns_is_refused(difr):
    buf = torch.zeros(4, 64, device=DEV)
    x, t, A = buf[:, 8:40], torch.zeros(4, dtype=torch.int32, device=DEV), torch.ones(4, device=DEV)
    off = torch.tensor([0, 2, 4], device=DEV)
    for call in (lambda V: difr.token_logprob(x, 1.0, t, V=V), lambda V: difr.policy_loss(x, 1.0, t, A, V=V),
                 lambda V: difr.preference_loss(x, 1.0, t, off, 0.1, V=V),
                 lambda V: difr.token_logprob_backward(x, 1.0, t, torch.ones(4, 2, device=DEV), A, V=V)):
        call(32), call(7)
        with pytest.raises(ValueError, match="V must be at most 32"):
            call(33)


def test_out_that_overlaps_is_refused(difr):
    buf = torch.zeros(10, 64, device=DEV)
    x, t = buf[:4], torch.zeros(4, dtype=torch.int32, device=DEV)
    A = torch.ones(4, device=DEV)
    for bad in (buf[1:5], buf[:4, :63], torch.zeros(4, 64, device=DEV).half(), torch.zeros(4, 64), torch.zeros(64, 4, device=DEV).t(),
                torch.zeros(1, 64, device=DEV).expand(4, 64)):
        with pytest.raises(ValueError, match="out must be"):
            difr.policy_loss(x, 1.0, t, A, out=bad)
    with pytest.raises(ValueError, match="advantages"):
        difr.policy_loss(x, 1.0, t, A.double())
    with pytest.raises(ValueError, match="advantages"):
        difr.policy_loss(x, 1.0, t, None)
    with pytest.raises(ValueError, match="seq_offsets"):
        difr.preference_loss(x, 1.0, t, torch.zeros(2, dtype=torch.int64, device=DEV), 0.1)
    with pytest.raises(ValueError, match="grad_entropy needs entropy"):
        difr.token_logprob_backward(x, 1.0, t, torch.zeros(4, 2, device=DEV), A, grad_entropy=A)
    with pytest.raises(difr.DifrError, match="temperature"):
        difr.policy_loss(x, 0.0, t, A)
    with pytest.raises(difr.DifrError, match="coefficient"):
        difr.policy_loss(x, 1.0, t, A, kl_coef=0.1)
