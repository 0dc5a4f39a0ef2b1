"""Operators on the logits of logged tokens - log-probabilities, losses with their gradients, and the product of a
head held in 4 bits - as cases that can be timed and compared.

Kinds (one of them per case):
  logp      token_logprob; with grad = 1 its gradient too, for upstream gradients of the log-probability and (entropy = 1)
            of the entropy
  policy    policy_loss with its gradient: the clipped ratio, a KL term against a reference policy, an entropy bonus
  pairs     preference_loss with its gradient: log ratios of chosen and rejected replies
  quantize  mx4_quantize, and back to values by mx4_dequantize
  product   hidden states quantised to 4 bits and multiplied by an LM-head matrix that is held in 4 bits

Logits have the value profile of ``paper_2511_02620_amd.workloads``: -1.1 ln(rank) in random order plus N(0,1).  Tokens are
drawn from them by the Gumbel-max sampler.  Where ``own`` is false, ``run`` computes the operators in elementary torch
operations in 32 bits; ``exact`` is their definition in 64 bits, row block by row block.
"""
import math
import random

import torch

own = False

DEV = "cuda"
BLOCK = 32                                           # elements that share a scale
SLAB = 128                                           # rows of codes are padded with zeros to whole slabs
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rows_case(name, kind, N, V, **kw):
    c = dict(name=name, kind=kind, N=N, V=V, dtype="bf16", T=1.0, row_T=0, pad=0, grad=1, entropy=0)
    if kind == "policy":
        c.update(masked=0.1, clip_low=0.2, clip_high=0.28, kl=0.02, bonus=0.0, drift=0.1)
    if kind == "pairs":
        c.update(pairs=2, masked=0.1, beta=0.1, smoothing=0.0, average=0)
    c.update(kw)
    return c


def listed():
    return [
        # the log-probabilities of one short reply, while the user waits
        _rows_case("logp_reply", "logp", 24, 151936, grad=0, entropy=1),
        # old and reference log-probabilities of a batch of replies, at the sampler's temperature
        _rows_case("logp_batch", "logp", 8192, 128256, grad=0, T=0.7),
        # a caller's own loss on log-probabilities and entropies, backward through both
        _rows_case("logp_train", "logp", 2048, 151936, entropy=1),
        # a toy vocabulary in fp32: launches are all there is
        _rows_case("policy_tiny", "policy", 64, 1024, dtype="f32"),
        # one step on 8 replies of 1024 tokens, prompt and padding left out
        _rows_case("policy_batch", "policy", 8192, 151936),
        # fp32 logits, a vocabulary that is no multiple of anything, a temperature of its own per request, an entropy bonus
        _rows_case("policy_odd", "policy", 1500, 99991, dtype="f32", row_T=1, bonus=0.01, entropy=1),
        # two pairs of short replies
        _rows_case("pairs_small", "pairs", 96, 50257),
        # 16 pairs of replies of some 250 tokens
        _rows_case("pairs_batch", "pairs", 8192, 128256, pairs=16, smoothing=0.1),
        # hidden states of the tokens that are decoded together
        dict(name="quantize_reply", kind="quantize", N=64, d=4096, dtype="bf16"),
        # an LM-head matrix, once when it is loaded
        dict(name="quantize_head", kind="quantize", N=151936, d=4096, dtype="bf16"),
        # logits of 16 tokens that are decoded together: the matrix is read for them
        dict(name="head_reply", kind="product", N=16, V=151936, d=4096, dtype="bf16", out="bf16"),
        # logits of four replies of 1024 tokens
        dict(name="head_batch", kind="product", N=4096, V=151936, d=4096, dtype="bf16", out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logp", "logp", "policy", "policy", "pairs", "quantize", "product", "product"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if kind == "quantize":
        return dict(kind=kind, N=_log_int(rng, 1, 32768), d=_log_int(rng, 16, 8192), dtype=dtype)
    V = _log_int(rng, 1000, 151936)
    if rng.random() < 0.5:
        V = -(-V // 64) * 64                         # half of the vocabularies are padded to 64, as served models' are
    if kind == "product":
        d = 32 * _log_int(rng, 8, 128) if rng.random() < 0.8 else _log_int(rng, 200, 4096)
        return dict(kind=kind, N=_log_int(rng, 1, 4096), V=V, d=d, dtype=dtype, out=rng.choice(["bf16", "bf16", "f32"]))
    N = _log_int(rng, 8 if kind == "pairs" else 1, 4096 if dtype == "f32" else 8192)
    kw = dict(dtype=dtype, T=round(rng.uniform(0.5, 1.3), 3), row_T=int(rng.random() < 0.3), entropy=int(rng.random() < 0.4))
    if rng.random() < 0.5:
        kw["pad"] = -V % 8                           # rows start on 16 bytes
    if kind == "logp":
        kw["grad"] = int(rng.random() < 0.6)
    if kind == "policy":
        kw.update(masked=round(rng.uniform(0.0, 0.5), 2), kl=rng.choice([0.0, 0.02, 0.1]), drift=round(rng.uniform(0.01, 0.3), 3),
                  bonus=0.01 if kw["entropy"] else 0.0)
    if kind == "pairs":
        kw.update(entropy=0, pairs=max(1, min(N // 4, _log_int(rng, 1, 32))), masked=round(rng.uniform(0.0, 0.5), 2),
                  beta=round(rng.uniform(0.05, 0.5), 2), smoothing=rng.choice([0.0, 0.1]), average=int(rng.random() < 0.3))
    c = _rows_case("", kind, N, V, **kw)
    del c["name"]
    return c


# ---- inputs -----------------------------------------------------------------------------------------------------

def _codes_of(x):
    """(codes, scales) of the rows of x: two 4-bit codes a byte, the lower half first; a scale byte per 32 elements."""
    codes, scales = [], []
    for r0 in range(0, x.shape[0], 16384):
        v, e = _split(x[r0:r0 + 16384])
        mag = v.abs()
        c = (mag > 0.25).to(torch.uint8)             # v is on the grid already: codes count the grid's points below it
        for edge in (0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
            c += mag > edge
        c += 8 * torch.signbit(v).to(torch.uint8)
        codes.append(c[:, 0::2] | (c[:, 1::2] << 4))
        scales.append((e + 127).to(torch.uint8))
    return torch.cat(codes), torch.cat(scales)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    N, kind, dtype = case["N"], case["kind"], DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    st = dict(case=dict(case))
    if kind in ("quantize", "product"):
        d = case["d"]
        size = (0.3 * normal(N, 1)).exp()            # rows of different size, a few large channels
        wide = 1 + 7 * (torch.rand(d, generator=g, device=DEV) < 0.01)
        st["hidden"] = (normal(N, d) * size * wide).to(dtype)
        if kind == "product":
            st["weight"] = _codes_of(normal(case["V"], d) / math.sqrt(d))
        return st

    V = case["V"]
    x = torch.rand(N, V, generator=g, device=DEV)
    x = x.mul_(V).add_(1).log_().mul_(-1.1).add_(normal(N, V))
    if case["pad"]:
        buf = torch.zeros(N, V + case["pad"], dtype=dtype, device=DEV)
        buf[:, :V] = x
        st["logits"] = buf[:, :V]
    else:
        st["logits"] = x.to(dtype)
    x = st["logits"].float()
    st["T"] = torch.rand(N, generator=g, device=DEV) * 0.8 + 0.5 if case["row_T"] else None
    x /= st["T"].unsqueeze(1) if case["row_T"] else case["T"]
    noise = torch.rand(N, V, generator=g, device=DEV).clamp_(1e-7, 1 - 1e-7).log_().neg_().log_().neg_()
    st["tokens"] = noise.add_(x).argmax(1).int()
    del noise
    if kind == "logp":
        if case["grad"]:
            st["grad_logp"] = normal(N) / N
            st["grad_entropy"] = 0.01 * normal(N) / N if case["entropy"] else None
        return st
    logp = x.gather(1, st["tokens"].long().unsqueeze(1)).squeeze(1) - x.logsumexp(1)
    keep = torch.rand(N, generator=g, device=DEV) >= case["masked"]
    keep[0] = True
    if kind == "policy":
        st["old"] = logp + case["drift"] * normal(N)
        st["ref"] = logp + 0.3 * normal(N) if case["kl"] else None
        st["advantages"] = normal(N)
        st["weights"] = keep.float() / max(1.0, float(keep.sum()))
        return st
    rng = random.Random(seed)
    S = 2 * case["pairs"]
    cuts = sorted(rng.sample(range(1, N), S - 1))
    st["offsets"] = torch.tensor([0] + cuts + [N], dtype=torch.int64, device=DEV)
    st["mask"] = keep.to(torch.uint8)
    total = torch.stack([s.mean() if case["average"] else s.sum() for s in (logp * keep).tensor_split(cuts)])
    st["ref"] = total + normal(S)
    return st


# ---- the plain form ---------------------------------------------------------------------------------------------

def _sequence_of(offsets, N):
    """The sequence of each of N rows."""
    return torch.searchsorted(offsets, torch.arange(N, device=offsets.device), right=True) - 1


def _softmax(st):
    """Of every row in 32 bits: (x - max) / T, the probabilities, log-probability of the token, entropy."""
    x = st["logits"].float()
    T = st["T"].unsqueeze(1) if st["T"] is not None else torch.full((1, 1), st["case"]["T"], device=DEV)
    y = (x - x.max(1, keepdim=True).values) / T
    del x
    p = y.exp()
    total = p.sum(1, keepdim=True)
    p /= total
    y -= total.log()                                 # now ln p
    logp = y.gather(1, st["tokens"].long().unsqueeze(1)).squeeze(1)
    entropy = -(p * y).sum(1) if st["case"]["entropy"] else None
    return y, p, logp, entropy, T


def _gradient(st, y, p, T, a, b, entropy):
    """d/dlogits for upstream gradients a of the log-probability and b of the entropy."""
    g = p * -a.unsqueeze(1)
    if b is not None:
        g -= b.unsqueeze(1) * p * (y + entropy.unsqueeze(1))
    g.scatter_add_(1, st["tokens"].long().unsqueeze(1), a.unsqueeze(1))
    return (g / T).to(st["logits"].dtype)


def _plain_logp(st):
    c = st["case"]
    y, p, logp, entropy, T = _softmax(st)
    out = dict(logp=logp)
    if c["entropy"]:
        out["entropy"] = entropy
    if c["grad"]:
        out["grad"] = _gradient(st, y, p, T, st["grad_logp"], st["grad_entropy"], entropy)
    return out


def _plain_policy(st):
    c = st["case"]
    y, p, logp, entropy, T = _softmax(st)
    A, w = st["advantages"], st["weights"]
    ratio = (logp - st["old"]).exp()
    inside = torch.minimum(torch.maximum(ratio, torch.full_like(ratio, 1 - c["clip_low"])), torch.full_like(ratio, 1 + c["clip_high"]))
    token_loss = -torch.minimum(ratio * A, inside * A)
    a = torch.where(ratio * A <= inside * A, -A * ratio, 0.0)
    if c["kl"]:
        d = st["ref"] - logp
        token_loss = token_loss + c["kl"] * (d.exp() - d - 1)
        a = a + c["kl"] * (1 - d.exp())
    if c["bonus"]:
        token_loss = token_loss - c["bonus"] * entropy
    live = w != 0
    zero = torch.zeros_like(w)
    out = dict(loss=(w.double() * token_loss).sum().float().reshape(1), token_loss=torch.where(live, token_loss, zero),
               logp=torch.where(live, logp, zero))
    out["grad"] = _gradient(st, y, p, T, w * a, -c["bonus"] * w if c["bonus"] else None, entropy)
    return out


def _plain_pairs(st):
    c = st["case"]
    y, p, logp, _, T = _softmax(st)
    keep = st["mask"] != 0
    S = 2 * c["pairs"]
    seq = _sequence_of(st["offsets"], c["N"])
    each = torch.where(keep, logp, torch.zeros_like(logp))
    total = torch.zeros(S, dtype=torch.float64, device=DEV).index_add_(0, seq, each.double())
    count = torch.zeros(S, dtype=torch.float64, device=DEV).index_add_(0, seq, keep.double())
    share = 1 / count.clamp(min=1) if c["average"] else torch.ones_like(count)
    total = total * share
    ratio = total - st["ref"].double()
    h = c["beta"] * (ratio[0::2] - ratio[1::2])
    eps = c["smoothing"]
    soft = torch.log1p((-h.abs()).exp())
    pair_loss = (1 - eps) * (soft + (-h).clamp(min=0)) + eps * (soft + h.clamp(min=0))
    up = 1 / (1 + (-h).exp())                        # sigma(h)
    dh = (eps * up - (1 - eps) * (1 - up)) * c["beta"] / c["pairs"]
    by_seq = torch.stack([dh, -dh], 1).reshape(-1) * share
    a = torch.where(keep, by_seq[seq], 0.0).float()
    return dict(loss=pair_loss.mean().float().reshape(1), pair_loss=pair_loss.float(), seq_logp=total.float(), logp=each,
                grad=_gradient(st, y, p, T, a, None, None))


def _split(x):
    """Elements on the grid of 4-bit floating point, and the exponent of each block's scale, of the rows of x; rows are padded with zeros."""
    N, d = x.shape
    K = -(-d // SLAB) * SLAB
    v = torch.zeros(N, K, device=x.device)
    v[:, :d] = x
    v = v.view(N, K // BLOCK, BLOCK)
    e = torch.frexp(v.abs().amax(2)).exponent - 3    # amax = m 2^f with m in [1/2, 1): floor(log2 amax) = f - 1
    e = torch.where(v.abs().amax(2) > 0, e, torch.full_like(e, -127)).clamp(min=-127)
    v = torch.ldexp(v, -e.unsqueeze(2))              # exact: a power of two
    mag = v.abs()
    step = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0))
    mag = ((mag / step).round() * step).clamp(max=6.0)
    return torch.copysign(mag, v).view(N, K), e


def _plain_quantize(st):
    v, e = _split(st["hidden"])
    N, d = st["hidden"].shape
    v = torch.ldexp(v.view(N, -1, BLOCK), e.unsqueeze(2)).view(N, -1)[:, :d]
    return v.to(torch.bfloat16)


_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _values_of(codes, scales):
    """The values that codes and scales stand for, in 32 bits."""
    grid = torch.tensor(_GRID + [-v for v in _GRID], device=codes.device)
    both = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], 1)     # the two values of a byte
    v = both[codes.long()].view(codes.shape[0], -1, BLOCK)
    return (v * torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127).unsqueeze(2)).view(codes.shape[0], -1)


def _plain_product(st):
    v, e = _split(st["hidden"])
    N = v.shape[0]
    a = torch.ldexp(v.view(N, -1, BLOCK), e.unsqueeze(2)).view(N, -1)
    return (a @ _values_of(*st["weight"]).t()).to(DTYPES[st["case"]["out"]])


# ---- one pass ---------------------------------------------------------------------------------------------------

def _own_pass(st):
    import paper_2511_02620_amd as difr

    c = st["case"]
    if c["kind"] == "quantize":
        q = difr.mx4_quantize(st["hidden"])
        return difr.mx4_dequantize(q["codes"], q["scales"], c["d"])
    if c["kind"] == "product":
        q = difr.mx4_quantize(st["hidden"])
        return difr.mx4_product(q["codes"], q["scales"], *st["weight"], dtype=DTYPES[c["out"]])
    at = (st["logits"], c["T"], st["tokens"])
    if c["kind"] == "logp":
        o = difr.token_logprob(*at, temperatures=st["T"], want_entropy=bool(c["entropy"]))
        out = {k: o[k] for k in ("logp", "entropy") if k in o}
        if c["grad"]:
            out["grad"] = difr.token_logprob_backward(*at, o["stats"], st["grad_logp"], entropy=o.get("entropy"),
                                                      grad_entropy=st["grad_entropy"], temperatures=st["T"])
        return out
    if c["kind"] == "policy":
        o = difr.policy_loss(*at, st["advantages"], st["weights"], old_logp=st["old"], ref_logp=st["ref"], clip_low=c["clip_low"],
                             clip_high=c["clip_high"], kl_coef=c["kl"], entropy_coef=c["bonus"], temperatures=st["T"])
        return {k: o[k] for k in ("loss", "token_loss", "logp", "grad")}
    o = difr.preference_loss(*at, st["offsets"], c["beta"], mask=st["mask"], ref_seq_logp=st["ref"],
                             label_smoothing=c["smoothing"], average=bool(c["average"]), temperatures=st["T"])
    return {k: o[k] for k in ("loss", "pair_loss", "seq_logp", "logp", "grad")}


def run(state):
    if own:
        return _own_pass(state)
    plain = {"logp": _plain_logp, "policy": _plain_policy, "pairs": _plain_pairs, "quantize": _plain_quantize,
             "product": _plain_product}
    return plain[state["case"]["kind"]](state)


def work(case):
    N, kind, size = case["N"], case["kind"], DTYPES[case["dtype"]].itemsize
    coded = 0.5 + 1 / BLOCK                          # bytes of an element in 4 bits with its share of the scale
    if kind == "quantize":
        return {"bytes": N * case["d"] * (size + coded + 2), "flops": 4 * N * case["d"]}
    if kind == "product":
        V, d = case["V"], case["d"]
        return {"bytes": N * d * size + V * d * coded + N * V * DTYPES[case["out"]].itemsize, "flops": 2 * N * V * d}
    V = case["V"]
    live = N * (1 - case.get("masked", 0.0))         # rows that count are read, gradients of all rows are written
    return {"bytes": live * V * size + (N * V * size if case["grad"] else 0) + 32 * N,
            "flops": live * V * (9 if case["grad"] else 5)}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def _exact_rows(st, upstream):
    """logp, entropy and gradient of all rows; upstream(logp, entropy) gives the two upstream gradients, or is None."""
    c = st["case"]
    x, N, V = st["logits"], c["N"], c["V"]
    T = st["T"].double() if st["T"] is not None else torch.full((N,), c["T"], dtype=torch.float32, device=DEV).double()
    chunk = max(1, (1 << 28) // V)
    logp = torch.empty(N, dtype=torch.float64, device=DEV)
    entropy = torch.empty(N, dtype=torch.float64, device=DEV)
    token = st["tokens"].long()
    for r in range(0, N, chunk):
        s = slice(r, min(N, r + chunk))
        lp = (x[s].double() / T[s, None]).log_softmax(1)
        logp[s] = lp[torch.arange(lp.shape[0], device=DEV), token[s]]
        entropy[s] = -(lp.exp() * lp).sum(1)
    if upstream is None:
        return logp, entropy, None
    a, b = upstream(logp, entropy)
    grad = torch.empty(N, V, dtype=x.dtype if x.dtype == torch.float32 else torch.float32, device=DEV)
    for r in range(0, N, chunk):
        s = slice(r, min(N, r + chunk))
        lp = (x[s].double() / T[s, None]).log_softmax(1)
        hot = torch.zeros_like(lp)
        hot[torch.arange(lp.shape[0], device=DEV), token[s]] = 1
        d = a[s, None] * (hot - lp.exp())
        if b is not None:
            d -= b[s, None] * lp.exp() * (lp + entropy[s, None])
        grad[s] = (d / T[s, None]).float()
    return logp, entropy, grad


def _exact_quantized(x):
    """The values that the rows of x have in 4 bits, in 64: the nearest point of the grid, ties to the even code."""
    N, d = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -d % BLOCK)).view(N, -1, BLOCK)
    top = v.abs().amax(2, keepdim=True)
    scale = 2.0 ** (top.clamp(min=2.0 ** -160).log2().floor() - 2).clamp(min=-127.0)
    scale = torch.where(scale * 8 <= top, scale * 2, torch.where(scale * 4 > top, scale / 2, scale)).clamp(min=2.0 ** -127)
    m = v.abs() / scale
    grid = torch.tensor(_GRID, dtype=torch.float64, device=DEV)
    best = torch.zeros_like(m)
    for k in range(1, 8):
        mid = (grid[k - 1] + grid[k]) / 2
        best = torch.where((m > mid) | ((m == mid) & (k % 2 == 0)), grid[k], best)
    return (best * scale * torch.sign(v)).view(N, -1)[:, :d]


def _exact_product(st):
    c = st["case"]
    K = st["weight"][0].shape[1] * 2
    a = torch.nn.functional.pad(_exact_quantized(st["hidden"]), (0, K - c["d"]))
    grid = torch.tensor(_GRID + [-v for v in _GRID], dtype=torch.float64, device=DEV)
    codes, scales = st["weight"]
    out = torch.empty(c["N"], c["V"], dtype=torch.float32, device=DEV)
    for v0 in range(0, c["V"], 16384):
        q = codes[v0:v0 + 16384]
        w = torch.empty(q.shape[0], K, dtype=torch.float64, device=DEV)
        w[:, 0::2] = grid[(q % 16).long()]
        w[:, 1::2] = grid[(q // 16).long()]
        w *= (2.0 ** (scales[v0:v0 + 16384].double() - 127)).repeat_interleave(BLOCK, 1)
        out[:, v0:v0 + q.shape[0]] = (a @ w.t()).float()
    return out


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        return torch.cat([_exact_quantized(st["hidden"][r:r + 16384]).float() for r in range(0, case["N"], 16384)])
    if kind == "product":
        return _exact_product(st)
    if kind == "logp":
        def upstream(logp, entropy):
            return st["grad_logp"].double(), None if st["grad_entropy"] is None else st["grad_entropy"].double()
        logp, entropy, grad = _exact_rows(st, upstream if case["grad"] else None)
        out = dict(logp=logp)
        if case["entropy"]:
            out["entropy"] = entropy
        if case["grad"]:
            out["grad"] = grad
        return out
    out = {}
    if kind == "policy":
        w, A = st["weights"].double(), st["advantages"].double()

        def upstream(logp, entropy):
            r = (logp - st["old"].double()).exp()
            cut = r.clamp(1 - case["clip_low"], 1 + case["clip_high"])
            clipped = r * A > cut * A
            loss = torch.where(clipped, -cut * A, -r * A)
            a = torch.where(clipped, torch.zeros_like(A), -r * A)
            if case["kl"]:
                d = st["ref"].double() - logp
                loss += case["kl"] * (torch.expm1(d) - d)
                a -= case["kl"] * torch.expm1(d)
            loss -= case["bonus"] * entropy
            out["loss"] = (w * loss).sum().reshape(1)
            out["token_loss"] = loss * (w != 0)
            out["logp"] = logp * (w != 0)
            return w * a, -case["bonus"] * w

        out["grad"] = _exact_rows(st, upstream)[2]
        return out
    keep = st["mask"].double()

    def upstream(logp, entropy):
        ends = st["offsets"].tolist()
        spans = [slice(a, b) for a, b in zip(ends[:-1], ends[1:])]
        div = [max(1.0, float(keep[s].sum())) if case["average"] else 1.0 for s in spans]
        total = torch.stack([(logp[s] * keep[s]).sum() / k for s, k in zip(spans, div)])
        ratio = total - st["ref"].double()
        h = case["beta"] * (ratio[0::2] - ratio[1::2])
        eps = case["smoothing"]
        ls = torch.nn.functional.logsigmoid
        loss = -(1 - eps) * ls(h) - eps * ls(-h)
        slope = (eps * torch.sigmoid(h) - (1 - eps) * torch.sigmoid(-h)) * case["beta"] / case["pairs"]
        a = torch.zeros_like(logp)
        for i, s in enumerate(spans):
            a[s] = keep[s] * slope[i // 2] * (1 - 2 * (i % 2)) / div[i]
        out.update(loss=loss.mean().reshape(1), pair_loss=loss, seq_logp=total, logp=logp * keep)
        return a, None

    out["grad"] = _exact_rows(st, upstream)[2]
    return out
