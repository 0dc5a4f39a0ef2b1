"""Verification of drafted tokens, in chains and in trees, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import draft_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def difr():
    import paper_2511_02620_amd as m
    m.load_library()
    return m


def _flags(difr):
    return difr.FLAG_MATCH, difr.FLAG_INVALID_CLAIM, difr.FLAG_NONFINITE


def _strided(t, pad, offset=0):
    N, V = t.shape
    buf = torch.full((offset + N * (V + pad),), math.nan, dtype=t.dtype, device=DEV)
    view = buf[offset:offset + N * (V + pad)].view(N, V + pad)[:, :V]
    view.copy_(t)
    return view


def _chains(seed, counts, V, dtype, drift=0.7, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    B, D = len(counts), sum(counts)
    offsets = [0]
    for c in counts:
        offsets.append(offsets[-1] + c)
    x = (torch.randn(D + B, V, generator=g) * spread).to(dtype)
    rows = [offsets[b] + b + i for b in range(B) for i in range(counts[b])]
    y = (x[rows].float() + drift * torch.randn(D, V, generator=g)).to(dtype)
    noise = -torch.log(-torch.log(torch.rand(D, V, generator=g).clamp(1e-7, 1 - 1e-7)))
    tokens = (y.float() + noise).argmax(1).int() if D else torch.zeros(0, dtype=torch.int32)
    return offsets, x, y, tokens, torch.rand(D, generator=g), torch.rand(B, generator=g)


def _agree(difr, got, want, names):
    for name, w in zip(names, want):
        v = got[name].cpu()
        if name == "logp":
            w = torch.tensor(w, dtype=torch.float64)
            # fp64 rounded once: half a step of fp32
            assert torch.equal(v.isnan(), w.isnan()), (name, v, w)
            off = (v.double() - w).abs().nan_to_num(0.0)
            assert (off <= w.abs().nan_to_num(0.0) * 2.0 ** -24 + 1e-14).all(), float(off.max())
        else:
            assert v.tolist() == list(w), (name, v.tolist(), w)


def _check_chain(difr, case, temperatures, draft_temperatures, with_draft=True, pad=0, offset=0, V=None):
    offsets, x, y, tokens, au, su = case
    R, D = x.shape[0], y.shape[0]
    T = temperatures if torch.is_tensor(temperatures) else torch.full((R,), temperatures)
    Td = draft_temperatures if torch.is_tensor(draft_temperatures) else torch.full((D,), draft_temperatures)
    n = x.shape[1] if V is None else V
    want = ref.draft_verify(x[:, :n], T.tolist(), tokens.tolist(), offsets, au.tolist(), su.tolist(), y[:, :n] if with_draft else None, Td.tolist(),
                            _flags(difr))
    kw = {}
    if torch.is_tensor(temperatures):
        kw.update(temperatures=T.to(DEV))
    if with_draft:
        kw.update(draft=_strided(y, pad, offset))
        if torch.is_tensor(draft_temperatures):
            kw.update(draft_temperatures=Td.to(DEV))
        else:
            kw.update(draft_temperature=draft_temperatures)
    got = difr.draft_verify(_strided(x, pad, offset), 1.0 if torch.is_tensor(temperatures) else temperatures, tokens.to(DEV),
                            torch.tensor(offsets).to(DEV), au.to(DEV), su.to(DEV), V=V, **kw)
    _agree(difr, got, want, ("accepted", "tokens", "logp", "flags"))
    return got, want


@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 1000, 2047, 2048, 2049, 4097, 50257])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,with_draft,pad,offset", [([4], True, 0, 0), ([0, 3, 1, 0, 5, 2], True, 3, 1), ([3, 0, 4], False, 1, 0), ([0], True, 0, 0),
                                                         ([0, 0, 0], False, 0, 0)])
def test_chains(difr, V, dtype, counts, with_draft, pad, offset):
    for seed in range(1 if V > 5000 else 3):
        _check_chain(difr, _chains(1000 * seed + V, counts, V, dtype), 0.8, 0.8, with_draft, pad, offset)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_chain_and_many_sequences(difr, dtype):
    got, _ = _check_chain(difr, _chains(3, [70], 300, dtype, drift=0.02), 1.0, 1.0)
    assert int(got["accepted"][0]) > 10
    got, _ = _check_chain(difr, _chains(4, [i % 6 for i in range(300)], 257, dtype, drift=0.5), 0.7, 0.9)
    assert 100 < int(got["accepted"].sum()) < 600
    # enough rows that a batch is no longer small
    got, _ = _check_chain(difr, _chains(5, [i % 5 for i in range(280)], 4100, dtype, drift=0.5), 1.1, 1.1)
    assert 100 < int(got["accepted"].sum()) < 500


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_temperatures_of_rows_and_drafts(difr, dtype):
    g = torch.Generator().manual_seed(8)
    case = _chains(11, [3, 4, 0, 2, 3, 3], 3000, dtype)
    T, Td = torch.rand(21, generator=g) + 0.4, torch.rand(15, generator=g) + 0.4
    _check_chain(difr, case, T, Td)
    _check_chain(difr, case, T, 0.6)
    _check_chain(difr, case, 0.5, Td, V=2900)
    for t in (1e-6, 1e-30, 1e6, 1e35):
        _check_chain(difr, _chains(12, [2, 3, 1], 500, dtype), t, t)


def test_a_draft_that_is_the_target_is_accepted_whole(difr):
    offsets, x, y, tokens, au, su = _chains(21, [5, 2, 8, 0], 3333, torch.bfloat16, drift=0.0)
    au = torch.full_like(au, 1 - 2.0 ** -24)
    got, _ = _check_chain(difr, (offsets, x, y, tokens, au, su), 0.8, 0.8)
    assert got["accepted"].tolist() == [5, 2, 8, 0]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masks(difr, dtype):
    low = float(torch.finfo(dtype).min)
    for mask in (-math.inf, low):
        offsets, x, y, tokens, au, su = _chains(31, [3, 3, 3, 3, 3, 3], 2500, dtype)
        g = torch.Generator().manual_seed(2)
        x[torch.rand(x.shape, generator=g) < 0.7] = mask
        y[torch.rand(y.shape, generator=g) < 0.5] = mask
        x[4], y[5] = mask, mask                           # rows without a finite logit (-inf), or uniform ones (lowest)
        x[8, :] = mask
        x[8, 2210] = 0.5                                  # one entry is all there is
        _check_chain(difr, (offsets, x, y, tokens, au, su), 0.9, 0.9)
        _check_chain(difr, (offsets, x, y, tokens, au, su), 0.9, 0.9, with_draft=False)


def test_a_masked_draft_under_the_same_distribution(difr):
    """p = q and the drafted token has no probability: nothing is left of p - q, so p is drawn from."""
    offsets, x, y, tokens, au, su = _chains(41, [1, 1], 700, torch.float32, drift=0.0)
    x[0, 5] = y[0, 5] = -math.inf
    x[2] += 3.0                                           # the same distribution by other logits
    x[2, 5] = y[1, 5] = -math.inf
    tokens[:] = 5
    got, want = _check_chain(difr, (offsets, x, y, tokens, au, su), 1.0, 1.0)
    assert got["accepted"].tolist() == [0, 0]


@pytest.mark.parametrize("bad", [math.nan, -math.nan, math.inf])
def test_rows_that_cannot_be_scored(difr, bad):
    for dtype in (torch.bfloat16, torch.float32):
        offsets, x, y, tokens, au, su = _chains(51, [4, 4, 4, 4], 2100, dtype, drift=0.0)
        au[:] = 0.999
        au[12] = 1.0 - 2.0 ** -24
        x[2, 2099] = bad                                  # of sequence 0, after two tokens
        y[5, 0] = bad                                     # of sequence 1, its second draft
        tokens[12] = -1                                   # sequence 3 does not come to the row after
        x[16, 77] = bad
        _check_chain(difr, (offsets, x, y, tokens, au, su), 1.0, 1.0)
        T = torch.ones(20)
        T[1], T[6], T[11], T[16] = 0.0, -1.0, math.nan, math.inf
        _check_chain(difr, _chains(52, [4, 4, 4, 4], 2100, dtype, drift=0.0), T, torch.ones(16))


def test_tokens_outside_and_numbers_outside(difr):
    offsets, x, y, tokens, au, su = _chains(61, [2, 2, 2, 2, 2, 2, 2], 1500, torch.bfloat16)
    tokens[0], tokens[2], tokens[5] = -1, 1500, 2 ** 31 - 1
    su[0], su[1], su[2], su[3], su[4] = math.nan, 1.0, -3.0, math.inf, 1.5
    au[7], au[9] = math.nan, math.inf
    _check_chain(difr, (offsets, x, y, tokens, au, su), 1.0, 1.0)
    _check_chain(difr, (offsets, x, y, tokens, au, su), 1.0, 1.0, with_draft=False)


def test_offsets_that_run_wild_stay_inside(difr):
    """What such offsets give is not defined, but every row that is read or written lies inside the tensors."""
    _, x, y, tokens, au, su = _chains(71, [3, 3, 3], 600, torch.float32)
    for off in ([0, 3, 6, 2 ** 40], [-5, 3, 6, 9], [0, 8, 2, 9], [2 ** 62, -2 ** 62, 4, 9], [9, 9, 9, 9]):
        got = difr.draft_verify(x.to(DEV), 1.0, tokens.to(DEV), torch.tensor(off).to(DEV), au.to(DEV), su.to(DEV), draft=y.to(DEV))
        tree = difr.tree_verify(x.to(DEV), 1.0, tokens.to(DEV), None, torch.tensor(off).to(DEV), torch.rand(12, device=DEV))
        torch.cuda.synchronize()
        assert got["accepted"].ge(0).all() and got["accepted"].le(9).all() and tree["accepted"].le(9).all()


def test_the_emitted_tokens_follow_the_target(difr):
    """20,000 sequences with one and the same target and a draft far from it: the first emitted token has the target's frequencies."""
    V, B = 6, 20000
    g = torch.Generator().manual_seed(5)
    p, q = torch.randn(V, generator=g), torch.randn(V, generator=g)
    draft = torch.multinomial(q.softmax(0), B, replacement=True, generator=g).int()
    off = torch.arange(B + 1).to(DEV)
    x, y = p.repeat(2 * B, 1).to(DEV), q.repeat(B, 1).to(DEV)
    n = {}
    for name, kw in (("draft", dict(draft=y)), ("lookup", {})):
        got = difr.draft_verify(x, 1.0, draft.to(DEV), off, torch.rand(B, generator=g).to(DEV), torch.rand(B, generator=g).to(DEV), **kw)
        n[name] = torch.bincount(got["tokens"][::2].cpu().long(), minlength=V)
    tree = difr.tree_verify(x, 1.0, draft.to(DEV), None, off, torch.rand(2 * B, generator=g).to(DEV))
    n["tree"] = torch.bincount(tree["tokens"][::2].cpu().long(), minlength=V)
    want = p.double().softmax(0) * B
    for name, count in n.items():
        assert ((count - want).abs() <= 5 * want.sqrt()).all(), (name, count, want)     # five standard deviations and more


# ---- trees ----

def _trees(seed, sizes, V, dtype, spread=2.0, fanout=3, hit=0.8):
    g = torch.Generator().manual_seed(seed)
    B, D = len(sizes), sum(sizes)
    offsets, parents = [0], []
    for n in sizes:
        offsets.append(offsets[-1] + n)
        parents += [max(-1, int(torch.randint(-1, j, (1,), generator=g)) if torch.rand(1, generator=g) < 0.5 else (j - 1) // fanout - (j > 0))
                    if j else -1 for j in range(n)]
    x = (torch.randn(D + B, V, generator=g) * spread).to(dtype)
    u = torch.rand(D + B, generator=g)
    tokens = torch.randint(0, V, (D,), generator=g, dtype=torch.int32)
    return offsets, parents, x, u, tokens, hit


def _hit(case, T, seed):
    """Some of the tokens that will be drawn go among the children of their rows, some of them twice."""
    offsets, parents, x, u, tokens, hit = case
    g = torch.Generator().manual_seed(seed)
    for b in range(len(offsets) - 1):
        k0, K = offsets[b], offsets[b + 1] - offsets[b]
        for at in range(-1, K):
            row = k0 + b + at + 1
            kids = [j for j in range(at + 1, K) if (j - 1 if parents is None else parents[k0 + j]) == at]
            if kids and torch.rand(1, generator=g) < hit:
                p = ref.probabilities(x[row], float(T[row]))
                t = ref.first_above(p, float(u[row])) if p is not None else 0
                for j in (kids[int(torch.randint(len(kids), (1,), generator=g))], kids[-1])[:1 + (at % 2)]:
                    tokens[k0 + j] = t


def _check_tree(difr, case, temperatures, pad=0, offset=0):
    offsets, parents, x, u, tokens, _ = case
    T = temperatures if torch.is_tensor(temperatures) else torch.full((x.shape[0],), temperatures)
    want = ref.tree_verify(x, T.tolist(), tokens.tolist(), parents, offsets, u.tolist(), _flags(difr))
    got = difr.tree_verify(_strided(x, pad, offset), 1.0 if torch.is_tensor(temperatures) else temperatures, tokens.to(DEV),
                           None if parents is None else torch.tensor(parents, dtype=torch.int32).to(DEV), torch.tensor(offsets).to(DEV), u.to(DEV),
                           temperatures=T.to(DEV) if torch.is_tensor(temperatures) else None)
    _agree(difr, got, want, ("accepted", "tokens", "nodes", "logp", "flags"))
    return got


@pytest.mark.parametrize("V", [1, 2, 8, 1000, 2049, 4097, 50257])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sizes,pad,offset", [([12], 0, 0), ([0, 5, 1, 30, 0], 3, 1), ([0], 0, 0)])
def test_trees(difr, V, dtype, sizes, pad, offset):
    for seed in range(1 if V > 5000 else 3):
        case = _trees(seed * 100 + V, sizes, V, dtype)
        _hit(case, torch.full((case[2].shape[0],), 0.9), seed)
        _check_tree(difr, case, 0.9, pad, offset)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_trees_chains_and_batches(difr, dtype):
    case = _trees(7, [150], 600, dtype, hit=0.95)
    _hit(case, torch.ones(151), 1)
    assert int(_check_tree(difr, case, 1.0)["accepted"][0]) >= 2
    case = _trees(8, [40, 25], 600, dtype, hit=1.0)
    case = (case[0], None) + case[2:]                                   # chains: each token follows the one before it
    _hit(case, torch.ones(67), 1)
    assert _check_tree(difr, case, 1.0)["accepted"].tolist() == [40, 25]
    T = torch.rand(300 + sum(i % 7 for i in range(300)), generator=torch.Generator().manual_seed(3)) + 0.5
    case = _trees(9, [i % 7 for i in range(300)], 2100, dtype)
    _hit(case, T, 2)
    assert int(_check_tree(difr, case, T)["accepted"].sum()) > 150


def test_trees_parents_that_are_no_parents(difr):
    case = _trees(14, [10, 10], 300, torch.float32, hit=1.0)
    parents = case[1]
    parents[3], parents[5], parents[12], parents[15] = 7, 5, -2, 2 ** 31 - 1        # later, itself, below the root, far away
    case = (case[0], parents) + case[2:]
    _hit(case, torch.ones(22), 1)
    _check_tree(difr, case, 1.0)


def test_trees_masks_and_rows_that_cannot_be_scored(difr):
    for dtype in (torch.bfloat16, torch.float32):
        for mask in (-math.inf, float(torch.finfo(dtype).min)):
            case = _trees(15, [8, 8, 8, 8], 2300, dtype, hit=1.0)
            x = case[2]
            x[torch.rand(x.shape, generator=torch.Generator().manual_seed(1)) < 0.6] = mask
            x[0] = mask
            x[10, :] = mask
            x[10, 2299] = -4.0
            x[19:22, 3] = math.nan
            x[28:31, 2] = math.inf
            _hit(case, torch.ones(36), 1)
            _check_tree(difr, case, 1.0)


def test_a_chain_without_a_draft_gives_what_the_sampler_draws(difr):
    """The tokens that verification emits with the seeded sampler's own uniforms are the sampler's tokens, and their scores match."""
    V, S, L = 5000, 6, 9
    g = torch.Generator().manual_seed(77)
    x = (torch.randn(S * L, V, generator=g) * 2).to(torch.bfloat16).to(DEV)
    seeds = torch.arange(1, S + 1, dtype=torch.int64, device=DEV) * 7919
    sid = torch.arange(S * L, device=DEV).div(L, rounding_mode="floor").int()
    pos = (torch.arange(S * L, device=DEV) % L).int()
    honest = difr.ipt_score(x, 0.8, seeds, sid, pos, None, want_token=True)
    off = torch.arange(S + 1, device=DEV) * (L - 1)
    tokens = honest["ipt_token"].view(S, L)[:, :L - 1].clone()
    tokens[2, 3] = (tokens[2, 3] + 1) % V                                # one draft is wrong
    got = difr.tree_verify(x, 0.8, tokens.reshape(-1).contiguous(), None, off, honest["u"])
    assert got["accepted"].tolist() == [L - 1, L - 1, 3, L - 1, L - 1, L - 1]
    emitted = got["tokens"].view(S, L)
    want = honest["ipt_token"].view(S, L).clone()
    want[2, 4:] = -1
    assert torch.equal(emitted, want)
    score = difr.ipt_score(x, 0.8, seeds, sid, pos, got["tokens"])
    assert (score["flags"].view(S, L)[emitted >= 0] & difr.FLAG_MATCH).all()


def test_a_serving_step_with_a_head_in_4_bits(difr):
    """Hidden states of drafted positions -> logits of a 4-bit head -> chains and trees, and the emitted tokens' log-probabilities."""
    V, d, counts = 3000, 512, [4, 4, 2, 0]
    B, D = len(counts), sum(counts)
    g = torch.Generator().manual_seed(3)
    q = difr.int4_quantize((torch.randn(V, d, generator=g) / 8).to(torch.bfloat16).to(DEV), group=64, zero_points=True)
    h = torch.randn(D + B, d, generator=g).to(torch.bfloat16).to(DEV)
    x = difr.int4_product(h, q["codes"], q["scales"], q["zeros"])
    off = torch.tensor([0, 4, 8, 10, 10], device=DEV)
    rows = torch.tensor([0, 1, 2, 3, 5, 6, 7, 8, 10, 11], device=DEV)
    y = (x[rows].float() + 0.3 * torch.randn(D, V, generator=g).to(DEV)).to(torch.bfloat16)
    tokens = (y.float() - torch.log(-torch.log(torch.rand(D, V, generator=g).clamp(1e-7, 1 - 1e-7).to(DEV)))).argmax(1).int()
    au, su = torch.rand(D, generator=g), torch.rand(B, generator=g)
    got = difr.draft_verify(x, 1.0, tokens, off, au.to(DEV), su.to(DEV), draft=y)
    want = ref.draft_verify(x.cpu(), [1.0] * (D + B), tokens.tolist(), off.tolist(), au.tolist(), su.tolist(), y.cpu(), [1.0] * D, _flags(difr))
    _agree(difr, got, want, ("accepted", "tokens", "logp", "flags"))
    out = got["tokens"]
    lp = difr.token_logprob(x, 1.0, out)["logp"]
    live = out >= 0
    assert (lp[live] - got["logp"][live]).abs().max() < 1e-5
    u = torch.rand(D + B, generator=g)
    tree = difr.tree_verify(x, 1.0, tokens, None, off, u.to(DEV))
    want = ref.tree_verify(x.cpu(), [1.0] * (D + B), tokens.tolist(), None, off.tolist(), u.tolist(), _flags(difr))
    _agree(difr, tree, want, ("accepted", "tokens", "nodes", "logp", "flags"))


def test_captured_and_replayed(difr):
    """A graph of a head, a chain and a tree, replayed with new inputs and eager work between the replays."""
    V, d, B, K = 4200, 256, 3, 4
    D = B * K
    g = torch.Generator().manual_seed(4)
    q = difr.int4_quantize((torch.randn(V, d, generator=g) / 8).to(DEV), group=32)
    off = torch.arange(B + 1, device=DEV) * K
    h = torch.empty(D + B, d, dtype=torch.bfloat16, device=DEV)
    y = torch.empty(D, V, device=DEV)
    tokens = torch.empty(D, dtype=torch.int32, device=DEV)
    au, su, u = torch.empty(D, device=DEV), torch.empty(B, device=DEV), torch.empty(D + B, device=DEV)

    def load(seed):
        g.manual_seed(seed)
        h.copy_(torch.randn(D + B, d, generator=g))
        for t in (au, su, u):
            t.copy_(torch.rand(t.shape, generator=g))
        x = difr.int4_product(h, q["codes"], q["scales"], dtype=torch.float32)
        rows = torch.arange(D, device=DEV) + torch.arange(D, device=DEV) // K
        y.copy_(x[rows] + 0.4 * torch.randn(D, V, generator=g).to(DEV))
        tokens.copy_(y.argmax(1))

    def step():
        x = difr.int4_product(h, q["codes"], q["scales"], dtype=torch.float32)
        return difr.draft_verify(x, 0.3, tokens, off, au, su, draft=y), difr.tree_verify(x, 0.3, tokens, None, off, u)

    load(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step()
    total = 0
    for seed in range(1, 6):
        load(seed)
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(recorded, eager):
            for k in a:
                assert torch.equal(a[k], b[k]), (seed, k)
        total += int(eager[0]["accepted"].sum()) + int(eager[1]["accepted"].sum())
    assert total > 0


def test_on_streams_of_their_own(difr):
    offsets, x, y, tokens, au, su = _chains(91, [4] * 8, 9000, torch.bfloat16, drift=0.4)
    args = (x.to(DEV), 1.0, tokens.to(DEV), torch.tensor(offsets).to(DEV), au.to(DEV), su.to(DEV))
    y = y.to(DEV)
    want = difr.draft_verify(*args, draft=y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    got = []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(difr.draft_verify(*args, draft=y))
    torch.cuda.synchronize()
    for o in got:
        assert all(torch.equal(o[k], want[k]) for k in want)


def test_draws_near_each_border(difr):
    """u at and beside the borders of the cumulative distribution, on rows of several cells."""
    V = 6000
    g = torch.Generator().manual_seed(13)
    x = (torch.randn(1, V, generator=g) * 2).to(torch.bfloat16)
    p = ref.probabilities(x[0], 1.0)
    c = np.cumsum(p)
    at = [0, 1, 2046, 2047, 2048, 2049, 4095, 4096, 4097, 5998]
    u = [float(np.float32(c[a])) for a in at] + [float(np.nextafter(np.float32(c[a]), np.float32(s))) for a in at for s in (0, 1)] + [0.0, 1 - 2.0 ** -24]
    want = [ref.first_above(p, v) for v in u]
    sure = [not ref.near(p, v, 1e-13) for v in u]
    assert sum(sure) >= len(u) - 2
    R = len(u)
    got = difr.tree_verify(x.repeat(R, 1).to(DEV), 1.0, torch.empty(0, dtype=torch.int32, device=DEV), None,
                           torch.zeros(R + 1, dtype=torch.int64, device=DEV), torch.tensor(u, dtype=torch.float32).to(DEV))["tokens"].tolist()
    assert [a for a, s in zip(got, sure) if s] == [a for a, s in zip(want, sure) if s]


@pytest.mark.parametrize("counts,drift,with_draft,dtype", [([3] * 140, 0.4, True, torch.bfloat16), ([i % 4 for i in range(150)], 0.5, True, torch.float32),
                                                           ([1] * 130 + [17], 0.02, True, torch.bfloat16),
                                                           ([i % 3 for i in range(270)], 0.0, False, torch.bfloat16)])
def test_large_batches_of_chains(difr, counts, drift, with_draft, dtype):
    """Batches that are taken level by level: chains of one length, of many, longer than the levels that are launched, and without drafts' logits."""
    V = 170000
    case = list(_chains(len(counts), counts, V, dtype, drift, spread=0.5 if with_draft else 6.0))
    if not with_draft:
        case[3] = case[2].float().argmax(1).int()                        # the likeliest token: such drafts stand now and then
    case[1][5] = math.nan                                                # some sequences end early
    case[3][4] = V + 7
    got, _ = _check_chain(difr, tuple(case), 0.9, 0.8 if drift > 0.1 else 0.9, with_draft)
    assert got["accepted"].max() >= min(2, max(counts))


@pytest.mark.parametrize("V", [40000, 70000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_batches_of_trees(difr, dtype, V):
    """All rows at once, and level by level."""
    case = _trees(17, [12, 0, 14, 13] * 22, V, dtype, hit=0.9)
    T = torch.rand(88 + 39 * 22, generator=torch.Generator().manual_seed(3)) + 0.5
    case[2][3] = math.nan
    _hit(case, T, 5)
    assert int(_check_tree(difr, case, T)["accepted"].max()) >= 3
    # chains deeper than the levels that are launched
    case = _trees(18, [10] * 90, V, dtype, hit=1.0)
    case = (case[0], None) + case[2:]
    _hit(case, torch.ones(990), 1)
    assert _check_tree(difr, case, 1.0)["accepted"].tolist() == [10] * 90


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [0.0625, 1.2890625, -3.0, 40.0])
def test_constant_rows_with_u_on_the_borders_of_cells(difr, dtype, value):
    """n tokens of one weight and u = k / 32: the definition is token k n / 32; a sum that is off in its last bit may stop at the one before,
    but nowhere else."""
    n, borders = 32 * 1024, torch.arange(32)
    u = (borders / 32).to(torch.float32).to(DEV)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    x = torch.full((32, n), value, dtype=dtype, device=DEV)
    off = torch.zeros(33, dtype=torch.int64, device=DEV)
    fits = [{k * 1024, max(k * 1024 - 1, 0)} for k in range(32)]

    def check(tokens):
        assert all(t in f for t, f in zip(tokens.tolist(), fits)), tokens.tolist()

    check(difr.tree_verify(x, 1.0, none, None, off, u)["tokens"])
    check(difr.draft_verify(x, 1.0, none, off, u[:0], u)["tokens"])
    # the rest of max(p - q, 0): the draft has only the tokens of a cell behind, one of which it proposes and which fall
    x = torch.full((64, n + 1024), value, dtype=dtype, device=DEV)
    y = torch.full((32, n + 1024), -math.inf, dtype=dtype, device=DEV)
    y[:, n:] = 1.0
    one = torch.arange(33, device=DEV)
    got = difr.draft_verify(x, 1.0, torch.full((32,), n + 5, dtype=torch.int32, device=DEV), one, torch.full((32,), 0.999, device=DEV), u, draft=y)
    assert got["accepted"].eq(0).all()
    check(got["tokens"][::2])
    # a draft without a distribution, in the last place
    got = difr.draft_verify(x[:, :n + 1], 1.0, torch.full((32,), n, dtype=torch.int32, device=DEV), one, torch.full((32,), 0.999, device=DEV), u)
    assert got["accepted"].eq(0).all()
    check(got["tokens"][::2])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("u", [0.0, -1.0, math.nan, 2.0 ** -24])
def test_tokens_of_hardly_any_probability(difr, dtype, u):
    """A running sum that exceeds 0 at entries of e^-624 and less, whole cells of which come first: they are drawn, masked ones never."""
    V, faint = 4 * 1024 + 9, -624.0
    x = torch.zeros(7, V)
    x[0, :1024] = faint
    x[1, :2048] = -680.0
    x[2, :1024], x[2, 1024:2048], x[2, 2048:2050], x[2, 2050:3072] = -math.inf, torch.finfo(dtype).min, -1e9, -680.0
    x[3, :5], x[3, 5:1024] = -1e9, faint
    x[4, :1500], x[4, 1500:] = faint, -math.inf
    x[4, 4104] = 0.0                                      # a single likely token, in the last cell
    x[5] = x[0] / 100.0
    x[6, :] = -math.inf
    x[6, 1024:2048], x[6, 3000], x[6, 4000] = -300.0, -950.0, -301.0
    x = x.to(dtype)
    T = torch.tensor([1.0, 1.0, 1.0, 1.0, 1.0, 0.01, 1.0])
    R = x.shape[0]
    us = torch.full((R,), u)
    none = torch.empty(0, dtype=torch.int32)
    off = [0] * (R + 1)
    names = ("accepted", "tokens", "logp", "flags")
    want = ref.tree_verify(x, T.tolist(), [], [], off, us.tolist(), _flags(difr))
    assert all(t >= 0 for t in want[1])
    d = lambda t: t.to(DEV)
    got = difr.tree_verify(d(x), 1.0, d(none), None, d(torch.tensor(off)), d(us), temperatures=d(T))
    _agree(difr, got, want, ("accepted", "tokens", "nodes", "logp", "flags"))
    want = ref.draft_verify(x, T.tolist(), [], off, [], us.tolist(), None, [], _flags(difr))
    _agree(difr, difr.draft_verify(d(x), 1.0, d(none), d(torch.tensor(off)), d(us[:0]), d(us), temperatures=d(T)), want, names)
    # a draft at every row: it falls, and what is left is drawn from
    off = list(range(R + 1))
    both = x.repeat_interleave(2, 0)
    T2 = T.repeat_interleave(2)
    y = both[::2].clone()
    y[:, V - 5:] = 0.0
    au = torch.full((R,), 0.99)
    for token in (V - 1, 0, 4104):
        tokens = torch.full((R,), token, dtype=torch.int32)
        for draft in (y, None):
            want = ref.draft_verify(both, T2.tolist(), tokens.tolist(), off, au.tolist(), us.tolist(), draft, T.tolist(), _flags(difr))
            got = difr.draft_verify(d(both), 1.0, d(tokens), d(torch.tensor(off)), d(au), d(us), draft=None if draft is None else d(draft),
                                    temperatures=d(T2), draft_temperatures=None if draft is None else d(T))
            _agree(difr, got, want, names)
    # trees whose drafts are no tokens at all
    tokens = torch.full((R,), -1, dtype=torch.int32)
    want = ref.tree_verify(both, T2.tolist(), tokens.tolist(), None, off, us.repeat_interleave(2).tolist(), _flags(difr))
    got = difr.tree_verify(d(both), 1.0, d(tokens), None, d(torch.tensor(off)), d(us.repeat_interleave(2)), temperatures=d(T2))
    _agree(difr, got, want, ("accepted", "tokens", "nodes", "logp", "flags"))
    assert got["accepted"].eq(0).all() and got["tokens"][::2].ge(0).all()


def test_numbers_outside_count_as_the_nearest_inside(difr):
    """sample_u: NaN and what is below as 0, what is above as 1 - 2^-24; accept_u: the same above and below (a NaN accepts nothing)."""
    V, big = 3000, 1 - 2.0 ** -24
    g = torch.Generator().manual_seed(6)
    x = torch.randn(12, V, generator=g)
    x[:, 2000:] = -40.0                                   # behind, tokens that no number below 1 - 2^-24 comes to
    x[:, 0] = -40.0
    d = lambda t: t.to(DEV)
    u = torch.tensor([0.0, math.nan, -0.5, -math.inf, big, 1.0, 1.5, math.inf, 0.5, 2.0 ** -149, -0.0, 1e30])
    same = [0, 0, 0, 0, 4, 4, 4, 4, 8, 9, 0, 4]
    one = d(x[:1].repeat(12, 1))
    none, off = torch.empty(0, dtype=torch.int32, device=DEV), torch.zeros(13, dtype=torch.int64, device=DEV)
    p = ref.probabilities(x[0], 1.0)
    assert 0 < ref.first_above(p, big) < 2000
    for got in (difr.tree_verify(one, 1.0, none, None, off, d(u)), difr.draft_verify(one, 1.0, none, off, none.float(), d(u))):
        t = got["tokens"].tolist()
        assert t == [t[i] for i in same] and t[0] == 0 and t[4] == ref.first_above(p, big)
    # p = q, by a draft and by a token that has all there is: only a NaN lets it fall
    x[1:] = x[:1]
    tokens, off = torch.full((12,), 7, dtype=torch.int32, device=DEV), torch.arange(13, device=DEV)
    rows = d(x[:1].repeat(24, 1))
    su = torch.full((12,), 0.5, device=DEV)
    stands = [0 if math.isnan(v) else 1 for v in u.tolist()]
    assert difr.draft_verify(rows, 1.0, tokens, off, d(u), su, draft=rows[:12])["accepted"].tolist() == stands
    rows[:] = -math.inf
    rows[:, 7] = 0.0
    assert difr.draft_verify(rows, 1.0, tokens, off, d(u), su)["accepted"].tolist() == stands


def test_a_draft_that_falls_where_nothing_is_left(difr):
    """p of the drafted token is 1 - 2^-50: what is left of p - q is below 2^-40, so p is drawn from, with a draft and without."""
    x = torch.full((2, 5), -math.inf)
    x[:, 1], x[:, 3] = 0.0, -50 * math.log(2.0)
    one, tokens = torch.tensor([0, 1]), torch.tensor([1], dtype=torch.int32)
    for draft in (None, torch.tensor([[-math.inf, 0.0, -math.inf, -math.inf, -math.inf]])):
        want = ref.draft_verify(x, [1.0, 1.0], [1], [0, 1], [math.nan], [0.5], draft, [1.0], _flags(difr))
        assert want[:2] == ([0], [1, -1])
        got = difr.draft_verify(x.to(DEV), 1.0, tokens.to(DEV), one.to(DEV), torch.full((1,), math.nan, device=DEV), torch.full((1,), 0.5, device=DEV),
                                draft=None if draft is None else draft.to(DEV))
        _agree(difr, got, want, ("accepted", "tokens", "logp", "flags"))


@pytest.mark.parametrize("V", [196609, 262144, 262145, 600000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_vocabularies(difr, V, dtype):
    """More cells than a wave holds of a row (192), and than are searched at once (256 of 1024 entries): draws in each round of the search, beside its
    border, and behind cells that are masked whole."""
    g = torch.Generator().manual_seed(V)
    T = float(torch.tensor(0.9))                          # as fp32 holds it
    x = (torch.randn(9, V, generator=g) * 2).to(dtype)
    edge = min(262144, V - 1025)
    x[3, :edge] = -math.inf
    x[4, :edge] = torch.finfo(dtype).min
    x[5, 1024:edge] = -math.inf
    x[6, :] = -math.inf
    x[6, edge], x[6, V - 1] = 0.0, 1.0
    x[7, 1024:] = -1e9
    x[8, :-1] = -math.inf
    us = []
    for row in range(9):
        p = ref.probabilities(x[row], T)
        c = np.cumsum(p)
        near_edge = [float(np.nextafter(np.float32(c[edge - 1]), np.float32(s))) for s in (0, 2)]
        us.append([u for u in [0.0, 0.31, 0.77, 1 - 2.0 ** -24] + near_edge if 0 <= u < 1 and not ref.near(p, u, 1e-12)])
        assert len(us[-1]) >= 2, row
    rows = [i for i in range(9) for _ in us[i]]
    flat = torch.tensor([u for row in us for u in row])
    R = len(rows)
    y, off, none = x[rows], [0] * (R + 1), torch.empty(0, dtype=torch.int32)
    want = ref.tree_verify(y, [T] * R, [], [], off, flat.tolist(), _flags(difr))
    args = (y.to(DEV), T, none.to(DEV))
    _agree(difr, difr.tree_verify(*args, None, torch.tensor(off).to(DEV), flat.to(DEV)), want, ("accepted", "tokens", "nodes", "logp", "flags"))
    want = want[:2] + want[3:]
    _agree(difr, difr.draft_verify(*args, torch.tensor(off).to(DEV), torch.empty(0, device=DEV), flat.to(DEV)), want, ("accepted", "tokens", "logp", "flags"))
    for with_draft in (True, False):
        case = _chains(V + 1, [2, 0, 1, 2], V, dtype)
        case[1][6, :edge], case[2][3, 7:edge] = -math.inf, -math.inf
        _check_chain(difr, case, 0.8, 0.8, with_draft)
    case = _trees(V + 2, [5, 3], V, dtype, hit=1.0)
    case[2][0, 5:edge] = -math.inf
    _hit(case, torch.ones(10), 1)
    assert int(_check_tree(difr, case, 1.0)["accepted"].sum()) >= 2


def test_large_batches_of_large_vocabularies(difr):
    """The same, level by level."""
    V = 300000
    case = _chains(5, [2] * 70, V, torch.bfloat16, drift=0.4, spread=1.0)
    case[1][::4, :262144] = -math.inf
    got, _ = _check_chain(difr, case, 0.9, 0.9)
    assert int(got["accepted"].sum()) > 30
    case = _trees(6, [6] * 30, V, torch.bfloat16, hit=1.0)
    case[2][::5, 100:262200] = -math.inf
    _hit(case, torch.ones(210), 2)
    assert int(_check_tree(difr, case, 1.0)["accepted"].sum()) > 30
