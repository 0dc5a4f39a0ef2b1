"""Operators of a server that decodes speculatively - the product of a few hidden states and a head held in 4-bit integers, and the
verification of drafted tokens, in chains and in trees - as cases that can be timed and compared.

Kinds (one of them per case):
  product   int4_product: hidden states by an LM-head matrix in 4-bit integers with a scale, and a zero point, for each group
  quantize  int4_quantize, and back to values by int4_dequantize
  draft     draft_verify: drafted tokens accepted or rejected by the ratio of the target's and the draft's probabilities (or, with
            lookup = 1, by the target's alone: the drafts come from a table), and the token that follows them
  tree      tree_verify: a token drawn at every row of the path that the drawn tokens take through a tree of drafted ones

Logits have the value profile of ``paper_2511_02620_amd.workloads``: -1.1 ln(rank) in random order plus N(0,1).  A draft's logits are the
target's plus ``drift`` N(0,1), its tokens are drawn from them.  Where ``own`` is false, ``run`` computes the operators in elementary torch
operations: products in 32 bits; probabilities and their sums, which decide whole numbers, in 64.  ``exact`` is their definition in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
SLAB = 128                                           # rows of codes are padded to whole slabs
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _draft_case(name, B, K, V, **kw):
    c = dict(name=name, kind="draft", B=B, K=K, V=V, dtype="bf16", T=1.0, row_T=0, ragged=0, lookup=0, drift=0.7, pad=0)
    c.update(kw)
    return c


def _tree_case(name, B, widths, V, **kw):
    c = dict(name=name, kind="tree", B=B, widths=widths, V=V, dtype="bf16", T=1.0, row_T=0, ragged=0, hit=0.7, pad=0)
    c.update(kw)
    return c


def listed():
    return [
        # one token of one request, a toy head in fp32: the launch is all there is
        dict(name="head_tiny", kind="product", N=1, V=1024, d=256, group=128, zeros=0, dtype="f32", out="f32"),
        # one token of one request: the head is read for it
        dict(name="head_token", kind="product", N=1, V=151936, d=4096, group=128, zeros=0, dtype="bf16", out="bf16"),
        # eight requests with four drafted tokens each
        dict(name="head_drafts", kind="product", N=40, V=128256, d=4096, group=64, zeros=1, dtype="bf16", out="bf16"),
        # nothing is a multiple of anything, fp32 logits
        dict(name="head_odd", kind="product", N=17, V=50257, d=2000, group=32, zeros=1, dtype="bf16", out="f32"),
        # one projection, and an LM-head matrix, once when they are loaded
        dict(name="quantize_small", kind="quantize", N=1024, d=4096, group=64, zeros=1, dtype="f32"),
        dict(name="quantize_head", kind="quantize", N=151936, d=4096, group=128, zeros=0, dtype="bf16"),
        # one request, four drafted tokens, while the user waits
        _draft_case("draft_reply", 1, 4, 151936),
        # a serving step: requests with up to five drafted tokens, a temperature each
        _draft_case("draft_step", 48, 5, 128256, row_T=1, ragged=1),
        # the largest: 256 requests, seven drafted tokens each
        _draft_case("draft_large", 256, 7, 151936, T=0.8),
        # drafts copied out of the prompt, fp32 logits, an odd vocabulary
        _draft_case("draft_lookup", 24, 6, 50257, dtype="f32", ragged=1, lookup=1, T=0.5),
        # one request with a tree of drafted tokens
        _tree_case("tree_reply", 1, "4,2,2,1", 151936),
        # requests with trees of different depth, logits that are padded to rows of whole lines
        _tree_case("tree_step", 64, "4,3,2,1", 128251, pad=5, ragged=1, row_T=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["product", "product", "product", "quantize", "draft", "draft", "draft", "tree", "tree"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    group, zeros = rng.choice([32, 64, 128]), int(rng.random() < 0.5)
    if kind == "quantize":
        return dict(kind=kind, N=_log_int(rng, 1, 32768), d=_log_int(rng, 16, 8192), group=group, zeros=zeros, dtype=dtype)
    V = _log_int(rng, 1000, 151936)
    if rng.random() < 0.5:
        V = -(-V // 64) * 64                         # half of the vocabularies are padded to 64, as served models' are
    if kind == "product":
        d = 32 * _log_int(rng, 8, 128) if rng.random() < 0.8 else _log_int(rng, 200, 4096)
        return dict(kind=kind, N=_log_int(rng, 1, 64), V=V, d=d, group=group, zeros=zeros, dtype=dtype, out=rng.choice(["bf16", "bf16", "f32"]))
    kw = dict(dtype=dtype, T=round(rng.uniform(0.5, 1.3), 3), row_T=int(rng.random() < 0.3), ragged=int(rng.random() < 0.5))
    if rng.random() < 0.5:
        kw["pad"] = -V % 8                           # rows start on 16 bytes
    if kind == "draft":
        K = rng.randint(0, 8)
        most = max(1, 280_000_000 // (V * (2 * K + 1)) // (2 if dtype == "f32" else 1))
        kw.update(lookup=int(rng.random() < 0.25), drift=round(rng.uniform(0.2, 1.2), 2))
        c = _draft_case("", _log_int(rng, 1, min(256, most)), K, V, **kw)
    else:
        widths = ",".join(str(rng.randint(1, 4)) for _ in range(rng.randint(1, 4)))
        rows = sum(_level_sizes(widths)) + 1
        most = max(1, 280_000_000 // (V * rows) // (2 if dtype == "f32" else 1))
        kw.update(hit=round(rng.uniform(0.3, 0.9), 2))
        c = _tree_case("", _log_int(rng, 1, min(128, most)), widths, V, **kw)
    del c["name"]
    return c


# ---- inputs -----------------------------------------------------------------------------------------------------

def _level_sizes(widths):
    """Nodes of each level of a tree in which every node of level i has widths[i] children."""
    sizes, n = [], 1
    for w in widths.split(","):
        n *= int(w)
        sizes.append(n)
    return sizes


def _parents(widths, depth):
    """The parent of each node, level by level; -1 is the root, whose children are the first level."""
    parents, level = [], [-1]
    for w in [int(w) for w in widths.split(",")][:depth]:
        first = len(parents)
        for node in level:
            parents += [node] * w
        level = list(range(first, len(parents)))
    return parents


def _shape(case):
    """Of each sequence its number of drafted tokens (or the depth of its tree): all there are, or any number up to that (the same ones
    in every pass over a case: they are the shape of its outputs)."""
    rng = random.Random(case["V"])
    most = case["K"] if case["kind"] == "draft" else len(case["widths"].split(","))
    return [rng.randint(0, most) if case["ragged"] else most for _ in range(case["B"])]


def _group_values(x, group, zeros):
    """Codes (0 to 15), scales and zero points of the rows of x, padded to whole slabs; 32 bits throughout, scales rounded to bf16."""
    N, d = x.shape
    K = -(-d // SLAB) * SLAB
    w = torch.zeros(N, K, device=x.device)
    w[:, :d] = x
    w = w.view(N, K // group, group)
    if zeros:
        lo, hi = w.amin(2).clamp(max=0.0), w.amax(2).clamp(min=0.0)
        scale = ((hi - lo) / torch.full_like(lo, 15)).to(torch.bfloat16)   # (a number would be multiplied by its inverse)
        s = scale.float()
        zero = torch.where(s > 0, (-lo / s).round().clamp(0, 15), torch.zeros_like(s))
    else:
        top = w.abs().amax(2)
        scale = (top / torch.full_like(top, 7)).to(torch.bfloat16)
        s = scale.float()
        zero = torch.full_like(s, 8.0)
    code = torch.where(s.unsqueeze(2) > 0, (w / s.unsqueeze(2)).round(), torch.zeros_like(w)) + zero.unsqueeze(2)
    return code.clamp(0, 15).view(N, K), scale, zero


def _coded(x, group, zeros):
    """What a program keeps of a matrix: two codes a byte, the lower half first; scales; zero points or None."""
    codes, scales, zs = [], [], []
    for r0 in range(0, x.shape[0], 16384):
        c, s, z = _group_values(x[r0:r0 + 16384], group, zeros)
        c = c.to(torch.uint8)
        codes.append(c[:, 0::2] | (c[:, 1::2] << 4))
        scales.append(s)
        zs.append(z.to(torch.uint8))
    return torch.cat(codes), torch.cat(scales), torch.cat(zs) if zeros else None


def _profile(rows, V, pad, dtype, normal, uniform):
    x = uniform(rows, V).mul_(V).add_(1).log_().mul_(-1.1).add_(normal(rows, V))
    buf = torch.zeros(rows, V + pad, dtype=dtype, device=DEV)
    buf[:, :V] = x
    return buf[:, :V]


def _drawn(x, T, u):
    """Tokens drawn by the Gumbel-max sampler from uniforms u."""
    return u.clamp_(1e-7, 1 - 1e-7).log_().neg_().log_().neg_().add_(x.float() / T).argmax(1).int()


def _by_chunk(rows, V):
    step = max(1, (1 << 27) // V)
    return [slice(r, min(rows, r + step)) for r in range(0, rows, step)]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=DEV)

    st = dict(case=dict(case))
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    if kind in ("quantize", "product"):
        N, d = case["N"], case["d"]
        size = (0.3 * normal(N, 1)).exp()            # rows of different size, a few large channels
        wide = 1 + 7 * (uniform(d) < 0.01)
        st["hidden"] = (normal(N, d) * size * wide).to(dtype)
        if kind == "product":
            st["weight"] = _coded(normal(case["V"], d) / math.sqrt(d), case["group"], case["zeros"])
        return st

    V, shape = case["V"], _shape(case)
    if kind == "tree":
        trees = [_parents(case["widths"], depth) for depth in shape]
        counts = [len(t) for t in trees]
    else:
        counts = shape
    B, D = case["B"], sum(counts)
    R = D + B
    ends = [0]
    for n in counts:
        ends.append(ends[-1] + n)
    st["offsets"] = torch.tensor(ends, dtype=torch.int64, device=DEV)
    st["logits"] = _profile(R, V, case["pad"], dtype, normal, uniform)
    # the row that each drafted token's predecessor has
    first = [ends[b] + b for b in range(B)]
    own_T = (uniform(B) * 0.8 + 0.5).tolist() if case["row_T"] else [case["T"]] * B
    of_row = [b for b in range(B) for _ in range(counts[b] + 1)]
    of_draft = [b for b in range(B) for _ in range(counts[b])]
    T = torch.tensor([own_T[b] for b in of_row], dtype=torch.float32, device=DEV)
    st["T"] = T if case["row_T"] else None
    if kind == "tree":
        st["parents"] = torch.tensor([p for t in trees for p in t], dtype=torch.int32, device=DEV)
        st["sample_u"] = uniform(R)
        # a draft that is right with probability `hit`: the token that will be drawn is among the children, the others are any
        will = torch.empty(R, dtype=torch.int32, device=DEV)
        for s in _by_chunk(R, V):
            will[s] = _inverse(st["logits"][s], T[s], st["sample_u"][s])
        lucky = (uniform(R) < case["hit"]).tolist()
        place, tokens, will = uniform(R).tolist(), torch.randint(V, (D,), generator=g, device=DEV, dtype=torch.int32).tolist(), will.tolist()
        for b in range(B):
            for slot in range(-1, counts[b]):
                kids = [j for j in range(slot + 1, counts[b]) if trees[b][j] == slot]
                row = first[b] + slot + 1
                if kids and lucky[row]:
                    tokens[ends[b] + kids[int(place[row] * len(kids))]] = will[row]
        st["tokens"] = torch.tensor(tokens, dtype=torch.int32, device=DEV)
        return st
    rows = torch.tensor([first[b] + i for b in range(B) for i in range(counts[b])], dtype=torch.int64, device=DEV)
    Td = torch.tensor([own_T[b] for b in of_draft], dtype=torch.float32, device=DEV)
    st["Td"] = Td if case["row_T"] else None
    buf = torch.zeros(D, V + case["pad"], dtype=dtype, device=DEV)
    st["draft"] = buf[:, :V]
    st["tokens"] = torch.empty(D, dtype=torch.int32, device=DEV)
    for s in _by_chunk(D, V):
        y = st["logits"][rows[s]].float()
        st["draft"][s] = y.add_(normal(*y.shape), alpha=case["drift"])
        st["tokens"][s] = _drawn(st["draft"][s], Td[s].unsqueeze(1), uniform(*y.shape))
    st["accept_u"], st["sample_u"] = uniform(D), uniform(B)
    if case["lookup"]:
        st["draft"] = None
    return st


# ---- the plain form ---------------------------------------------------------------------------------------------

def _inverse(x, T, u):
    """min{v: C_v > u} of softmax(x / T), in 64 bits."""
    p = x.double() / T.double().unsqueeze(1)
    p = (p - p.amax(1, keepdim=True)).exp().cumsum(1)
    return (p <= u.double().unsqueeze(1) * p[:, -1:]).sum(1).clamp(max=x.shape[1] - 1).int()


def _temperature(st, key, rows):
    return st[key] if st[key] is not None else torch.full((rows,), st["case"]["T"], device=DEV)


def _log_z(x, T):
    """ln sum exp(x / T) of every row, in 64 bits."""
    out = torch.empty(x.shape[0], dtype=torch.float64, device=x.device)
    for s in _by_chunk(*x.shape):
        y = x[s].double() / T[s].double().unsqueeze(1)
        top = y.amax(1)
        out[s] = (y - top.unsqueeze(1)).exp().sum(1).log() + top
    return out


def _at(x, T, logz, tokens):
    """ln softmax(x / T) of each row's token."""
    return x.gather(1, tokens.long().unsqueeze(1)).squeeze(1).double() / T.double() - logz


def _plain_draft(st):
    x, y, off, tokens = st["logits"], st["draft"], st["offsets"], st["tokens"]
    B, D, R = off.shape[0] - 1, tokens.shape[0], x.shape[0]
    T, count = _temperature(st, "T", R), off[1:] - off[:-1]
    first = off[:-1] + torch.arange(B, device=DEV)                   # first row of each sequence
    of_draft = torch.repeat_interleave(torch.arange(B, device=DEV), count)
    place = torch.arange(D, device=DEV) - off[of_draft]              # of each drafted token in its sequence
    row = first[of_draft] + place
    logz = _log_z(x, T)
    lp = _at(x[row], T[row], logz[row], tokens)
    if y is None:
        q, Td, logzd = torch.ones(D, dtype=torch.float64, device=DEV), None, None
    else:
        Td = _temperature(st, "Td", D)
        logzd = _log_z(y, Td)
        q = _at(y, Td, logzd, tokens).exp()
    falls = ~(st["accept_u"].double() * q < lp.exp())
    accepted = count.clone()
    accepted.scatter_reduce_(0, of_draft[falls], place[falls], "amin")
    stop = first + accepted
    drawn = torch.empty(B, dtype=torch.int64, device=DEV)
    for s in _by_chunk(B, x.shape[1]):
        p = (x[stop[s]].double() / T[stop[s]].double().unsqueeze(1) - logz[stop[s]].unsqueeze(1)).exp()
        fell = (accepted[s] < count[s]).nonzero().squeeze(1)
        at = (off[:-1][s] + accepted[s])[fell]
        if y is None:
            r = p[fell]
            r[torch.arange(fell.shape[0], device=DEV), tokens[at].long()] = 0
        else:
            r = (p[fell] - (y[at].double() / Td[at].double().unsqueeze(1) - logzd[at].unsqueeze(1)).exp()).clamp(min=0)
        p[fell] = torch.where(r.sum(1, keepdim=True) > 0, r, p[fell])
        c = p.cumsum(1)
        drawn[s] = (c <= st["sample_u"][s].double().unsqueeze(1) * c[:, -1:]).sum(1).clamp(max=x.shape[1] - 1)
    out = torch.full((R,), -1, dtype=torch.int32, device=DEV)
    logp = torch.zeros(R, device=DEV)
    kept = place < accepted[of_draft]
    out[row[kept]] = tokens[kept]
    logp[row[kept]] = lp[kept].float()
    out[stop] = drawn.int()
    logp[stop] = _at(x[stop], T[stop], logz[stop], drawn).float()
    return dict(accepted=accepted.int(), tokens=out, logp=logp)


def _plain_tree(st):
    x, off, tokens, parents = st["logits"], st["offsets"], st["tokens"], st["parents"]
    B, D, R = off.shape[0] - 1, tokens.shape[0], x.shape[0]
    T, count = _temperature(st, "T", R), off[1:] - off[:-1]
    first = off[:-1] + torch.arange(B, device=DEV)
    node = torch.arange(D, device=DEV)
    of_draft = torch.repeat_interleave(torch.arange(B, device=DEV), count)
    out = torch.full((R,), -1, dtype=torch.int32, device=DEV)
    nodes, logp = out.clone(), torch.zeros(R, device=DEV)
    accepted = torch.zeros(B, dtype=torch.int64, device=DEV)
    at = torch.full((B,), -1, dtype=torch.int64, device=DEV)         # the node where each sequence is
    going = torch.ones(B, dtype=torch.bool, device=DEV)
    for _ in range(len(st["case"]["widths"].split(",")) + 1):
        row = first + at + 1
        drawn = torch.zeros(B, dtype=torch.int32, device=DEV)
        lp = torch.zeros(B, device=DEV)
        for s in _by_chunk(B, x.shape[1]):
            xs, Ts = x[row[s]], T[row[s]]
            drawn[s] = _inverse(xs, Ts, st["sample_u"][row[s]])
            lp[s] = _at(xs, Ts, _log_z(xs, Ts), drawn[s]).float()
        active = going.nonzero().squeeze(1)
        to = (first + accepted)[active]
        out[to], logp[to] = drawn[active], lp[active]
        fits = (parents == at[of_draft]) & (tokens == drawn[of_draft]) & going[of_draft]
        child = torch.full((B,), D, dtype=torch.int64, device=DEV)   # the first child that holds the drawn token
        child.scatter_reduce_(0, of_draft[fits], (node - off[of_draft])[fits], "amin")
        going = child < D
        nodes[to] = torch.where(going, child, -1).int()[active]
        accepted = accepted + going.long()
        at = torch.where(going, child, at)
    return dict(accepted=accepted.int(), tokens=out, nodes=nodes, logp=logp)


def _values(codes, scales, zeros):
    """The values that codes, scales and zero points stand for, in 32 bits."""
    both = torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], scales.shape[1], -1).float()
    return ((both - (8.0 if zeros is None else zeros.float().unsqueeze(2))) * scales.float().unsqueeze(2)).view(codes.shape[0], -1)


def _plain_product(st):
    h = st["hidden"].float()
    codes, scales, zeros = st["weight"]
    out = [h @ _values(codes[v:v + 32768], scales[v:v + 32768], None if zeros is None else zeros[v:v + 32768])[:, :h.shape[1]].t()
           for v in range(0, codes.shape[0], 32768)]
    return torch.cat(out, 1).to(DTYPES[st["case"]["out"]])


def _plain_quantize(st):
    x, c = st["hidden"], st["case"]
    out = []
    for r in range(0, x.shape[0], 32768):
        code, scale, zero = _group_values(x[r:r + 32768], c["group"], c["zeros"])
        v = (code.view(*scale.shape, -1) - zero.unsqueeze(2)) * scale.float().unsqueeze(2)
        out.append(v.view(v.shape[0], -1)[:, :c["d"]])
    return torch.cat(out).contiguous()


# ---- one pass ---------------------------------------------------------------------------------------------------

def _own_pass(st):
    import paper_2511_02620_amd as difr

    c = st["case"]
    if c["kind"] == "product":
        codes, scales, zeros = st["weight"]
        return difr.int4_product(st["hidden"], codes, scales, zeros, dtype=DTYPES[c["out"]])
    if c["kind"] == "quantize":
        q = difr.int4_quantize(st["hidden"], group=c["group"], zero_points=bool(c["zeros"]))
        return difr.int4_dequantize(q["codes"], q["scales"], c["d"], q.get("zeros"), dtype=torch.float32)
    if c["kind"] == "draft":
        o = difr.draft_verify(st["logits"], c["T"], st["tokens"], st["offsets"], st["accept_u"], st["sample_u"], draft=st["draft"],
                              temperatures=st["T"], draft_temperatures=None if st["draft"] is None else st["Td"])
        return {k: o[k] for k in ("accepted", "tokens", "logp")}
    o = difr.tree_verify(st["logits"], c["T"], st["tokens"], st["parents"], st["offsets"], st["sample_u"], temperatures=st["T"])
    return {k: o[k] for k in ("accepted", "tokens", "nodes", "logp")}


def run(state):
    if own:
        return _own_pass(state)
    plain = {"product": _plain_product, "quantize": _plain_quantize, "draft": _plain_draft, "tree": _plain_tree}
    return plain[state["case"]["kind"]](state)


def work(case):
    kind, size = case["kind"], DTYPES[case["dtype"]].itemsize
    if kind in ("product", "quantize"):
        N, d = case["N"], case["d"]
        coded = 0.5 + (2 + case["zeros"]) / case["group"]            # bytes of an element with its share of scale and zero point
        if kind == "quantize":
            return {"bytes": N * d * (size + coded + 4), "flops": 6 * N * d}
        V = case["V"]
        return {"bytes": N * d * size + V * d * coded + N * V * DTYPES[case["out"]].itemsize, "flops": 2 * N * V * d}
    # the rows that decide: those up to where a sequence stops, as many as are expected
    V, B = case["V"], case["B"]
    if kind == "draft":
        most = case["K"]
        stays = 0.4 if case["lookup"] else math.erfc(case["drift"] / math.sqrt(8))
        both = 0 if case["lookup"] else 1
    else:
        most, stays, both = len(case["widths"].split(",")), case["hit"], 0
    rows = 0.0
    for length in (range(most + 1) if case["ragged"] else [most]):
        reached = [stays ** i for i in range(length + 1)]
        rows += sum(reached) + both * sum(reached[:-1])
    rows *= B / (most + 1 if case["ragged"] else 1)
    return {"bytes": rows * V * size + 16 * B, "flops": rows * V * 20}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def _exact_product(st):
    codes, scales, zeros = st["weight"]
    h = st["hidden"].double()
    K = 2 * codes.shape[1]
    group = K // scales.shape[1]
    out = torch.empty(h.shape[0], codes.shape[0], dtype=torch.float64, device=DEV)
    for v in range(0, codes.shape[0], 8192):
        w = torch.empty(min(8192, codes.shape[0] - v), K, dtype=torch.float64, device=DEV)
        w[:, 0::2] = (codes[v:v + 8192] % 16).double()
        w[:, 1::2] = (codes[v:v + 8192] // 16).double()
        w -= 8 if zeros is None else zeros[v:v + 8192].double().repeat_interleave(group, 1)
        w *= scales[v:v + 8192].double().repeat_interleave(group, 1)
        out[:, v:v + 8192] = h @ w[:, :h.shape[1]].t().contiguous()
    return out


def _exact_quantize(x, group, zeros):
    """Scales are quotients in 32 bits rounded to bf16, codes quotients in 32 bits rounded to whole numbers: that is the definition."""
    out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    d = x.shape[1]
    for k in range(0, d, group):
        w = x[:, k:k + group].double()
        if zeros:
            lo, hi = w.min(1).values.clamp(max=0), w.max(1).values.clamp(min=0)
            s = ((hi - lo).float().double() / 15).float().bfloat16().double()
            z = (-lo / s.where(s > 0, torch.ones_like(s))).float().double().round().clamp(0, 15) * (s > 0)
        else:
            s = (w.abs().max(1).values / 7).float().bfloat16().double()
            z = torch.full_like(s, 8)
        n = (w / s.where(s > 0, torch.ones_like(s)).unsqueeze(1)).float().double().round() * (s > 0).unsqueeze(1)
        n = torch.minimum(torch.maximum(n, -z.unsqueeze(1)), 15 - z.unsqueeze(1))
        out[:, k:k + group] = n * s.unsqueeze(1)
    return out


def _exact_probabilities(row, T):
    return torch.softmax(row.double() / float(T), 0)


def _exact_token(weights, u):
    """The first token whose cumulative weight is above u times the whole."""
    c = torch.cumsum(weights, 0)
    return min(int(torch.searchsorted(c, c[-1:] * float(u), right=True)), weights.shape[0] - 1)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "product":
        return _exact_product(st)
    if case["kind"] == "quantize":
        return _exact_quantize(st["hidden"], case["group"], case["zeros"])
    x, ends, tokens = st["logits"], st["offsets"].tolist(), st["tokens"].tolist()
    one = float(torch.tensor(case["T"], dtype=torch.float32))
    T = st["T"].tolist() if st["T"] is not None else [one] * x.shape[0]
    u = st["sample_u"].tolist()
    accepted, emitted, nodes, logp = [], [-1] * x.shape[0], [-1] * x.shape[0], [0.0] * x.shape[0]
    for b in range(case["B"]):
        row0, mine = ends[b] + b, tokens[ends[b]:ends[b + 1]]
        if case["kind"] == "tree":
            parents = st["parents"][ends[b]:ends[b + 1]].tolist()
            at, n = -1, 0
            while True:
                p = _exact_probabilities(x[row0 + at + 1], T[row0 + at + 1])
                t = _exact_token(p, u[row0 + at + 1])
                emitted[row0 + n], logp[row0 + n] = t, math.log(float(p[t]))
                kids = [j for j, (q, token) in enumerate(zip(parents, mine)) if q == at and token == t]
                if not kids:
                    break
                at = nodes[row0 + n] = kids[0]
                n += 1
            accepted.append(n)
            continue
        n, weights = 0, None
        while True:
            p = _exact_probabilities(x[row0 + n], T[row0 + n])
            if n == len(mine):
                weights = p
                break
            k = ends[b] + n
            if st["draft"] is None:
                q = torch.zeros_like(p)
                q[mine[n]] = 1
            else:
                q = _exact_probabilities(st["draft"][k], st["Td"][k] if st["Td"] is not None else one)
            if float(st["accept_u"][k]) * float(q[mine[n]]) < float(p[mine[n]]):
                emitted[row0 + n], logp[row0 + n] = mine[n], math.log(float(p[mine[n]]))
                n += 1
                continue
            weights = (p - q).clamp(min=0)
            if float(weights.sum()) <= 0:
                weights = p
            break
        t = _exact_token(weights, u[b])
        emitted[row0 + n], logp[row0 + n] = t, math.log(float(p[t]))
        accepted.append(n)

    def whole(v):
        return torch.tensor(v, dtype=torch.int32, device=DEV)

    out = dict(accepted=whole(accepted), tokens=whole(emitted))
    if case["kind"] == "tree":
        out["nodes"] = whole(nodes)
    out["logp"] = torch.tensor(logp, dtype=torch.float64, device=DEV)
    return out
