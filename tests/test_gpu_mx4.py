"""Microscaled 4-bit floating point against its definition in 64 bits: codes, values, products, and a head in 4 bits under the scores and
a loss."""
import math

import pytest
import torch

import token_loss_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def difr():
    import paper_2511_02620_amd as m
    m.load_library()
    return m


def _same(a, b):
    return torch.equal(a.cpu().double().nan_to_num(nan=-77.0), b.double().nan_to_num(nan=-77.0))


@pytest.mark.parametrize("N,d", [(1, 1), (3, 31), (2, 32), (5, 33), (4, 127), (3, 128), (2, 129), (7, 1000), (33, 4096), (300, 40)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset,gap", [(0, 0), (1, 0), (5, 3)])
def test_quantize_and_back(difr, N, d, dtype, offset, gap):
    g = torch.Generator().manual_seed(N * 100 + d)
    x = (torch.randn(N, d, generator=g) * (4 * torch.randn(N, 1, generator=g)).exp()).to(dtype)
    buf = torch.full((offset + N * (d + gap),), math.nan, dtype=dtype, device=DEV)      # what lies between the rows is not read
    view = buf[offset:].view(N, d + gap)[:, :d]
    view.copy_(x)
    codes, scales, values = ref.mx4(x)
    q = difr.mx4_quantize(view)
    assert torch.equal(q["codes"].cpu(), codes) and torch.equal(q["scales"].cpu(), scales)
    for out in (torch.bfloat16, torch.float32):
        back = difr.mx4_dequantize(q["codes"], q["scales"], d, dtype=out)
        assert back.dtype == out and _same(back, values[:, :d])


def test_ties_edges_and_what_is_no_number(difr):
    for dtype in (torch.float32, torch.bfloat16):
        half = torch.arange(-64, 64).double() / 16              # all ties and what lies between them
        rows = [half[:32], half[32:64], half[64:96], half[96:]]
        big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).tiny
        for k in (-140, -133, -127, -126, -125, -124, -120, 0, 60, 120, 125):
            rows.append(half[96:] * 2.0 ** k)
        rows += [torch.zeros(32).double(), -torch.zeros(32).double(), torch.full((32,), big).double(), torch.full((32,), -tiny).double()]
        for bad in (math.nan, math.inf, -math.inf):
            r = half[:32].clone()
            r[7] = bad
            rows.append(r)
        x = torch.stack(rows).to(dtype)
        x = torch.cat([x, x.flip(0)], 1)                          # a bad block leaves its neighbours alone
        codes, scales, values = ref.mx4(x)
        q = difr.mx4_quantize(x.to(DEV))
        assert torch.equal(q["scales"].cpu(), scales), dtype
        assert torch.equal(q["codes"].cpu(), codes), dtype
        assert _same(difr.mx4_dequantize(q["codes"], q["scales"], 64, dtype=torch.float32), values[:, :64])


def _operands(seed, N, V, d):
    g = torch.Generator().manual_seed(seed)
    a = torch.randn(N, d, generator=g) * (2 * torch.randn(N, 1, generator=g)).exp()
    b = torch.randn(V, d, generator=g) / math.sqrt(d)
    return a, b


def _bound(a, b, want, dtype):
    """The products are exact in fp32 and a sum of K of them is off by at most K half steps of the sum of magnitudes (whatever the order);
    the result is rounded once."""
    size = a.abs() @ b.abs().t()
    return ref.EPS[dtype] * want.abs() + 2.0 ** -24 * a.shape[1] * size


@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 33, 64, 65, 127, 130, 200, 256, 257, 515])
@pytest.mark.parametrize("V,d", [(1, 128), (100, 40), (257, 384), (1000, 1000), (515, 4096), (4111, 256)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_product(difr, N, V, d, dtype):
    a, b = _operands(N * 7 + V, N, V, d)
    va, vb = ref.mx4(a)[2], ref.mx4(b)[2]
    want = va @ vb.t()
    qa, qb = difr.mx4_quantize(a.to(DEV)), difr.mx4_quantize(b.to(DEV))
    args = (qa["codes"], qa["scales"], qb["codes"], qb["scales"])
    got = difr.mx4_product(*args, dtype=dtype)
    assert got.dtype == dtype and got.shape == (N, V)
    ref.assert_within(got, want, _bound(va, vb, want, dtype), "product")
    buf = torch.full((N + 1, V + 3), 7.0, dtype=dtype, device=DEV)
    into = buf[:N, 1:V + 1]
    difr.mx4_product(*args, dtype=dtype, out=into)
    assert torch.equal(into, got), "into a view"
    assert buf[N].eq(7).all() and buf[:, 0].eq(7).all() and buf[:, V + 1:].eq(7).all(), "what lies around it"


def test_product_of_extreme_scales_and_nan(difr):
    a = torch.ones(20, 256)
    b = torch.ones(40, 256)
    a[1] *= 2.0 ** 100
    a[2] *= 2.0 ** -126
    b[1] *= 2.0 ** -100
    b[2] *= 2.0 ** 20
    a[3, 40], b[3, 200] = math.nan, math.inf
    a[4, :128] = 0
    va, vb = ref.mx4(a)[2], ref.mx4(b)[2]
    qa, qb = difr.mx4_quantize(a.to(DEV)), difr.mx4_quantize(b.to(DEV))
    got = difr.mx4_product(qa["codes"], qa["scales"], qb["codes"], qb["scales"], dtype=torch.float32)
    want = va @ vb.t()
    # (2^-126 2^-100 256 = 2^-218 has no place in fp32: what is below its smallest normal number, 2^-126, may come out as 0)
    ref.assert_within(got, want, 2.0 ** -24 * 256 * want.abs().nan_to_num(0) + 2.0 ** -126, "product")


def test_no_rows(difr):
    e = torch.zeros(0, 300, device=DEV)
    q = difr.mx4_quantize(e)
    assert q["codes"].shape == (0, 192) and q["scales"].shape == (0, 12)
    assert difr.mx4_dequantize(q["codes"], q["scales"], 300).shape == (0, 300)
    w = difr.mx4_quantize(torch.ones(5, 300, device=DEV))
    assert difr.mx4_product(q["codes"], q["scales"], w["codes"], w["scales"]).shape == (0, 5)
    assert difr.mx4_product(w["codes"], w["scales"], q["codes"], q["scales"]).shape == (5, 0)


def test_what_is_refused(difr):
    q = difr.mx4_quantize(torch.ones(5, 300, device=DEV))
    w = difr.mx4_quantize(torch.ones(5, 100, device=DEV))
    c, s = q["codes"], q["scales"]
    with pytest.raises(ValueError, match="rows as long"):
        difr.mx4_product(c, s, w["codes"], w["scales"])
    for bad in (c[:, :100], c.int(), c.t(), c[0], c[:, :-16]):
        with pytest.raises(ValueError, match="codes must be"):
            difr.mx4_product(bad, s, c, s)
    with pytest.raises(ValueError, match="scales must be"):
        difr.mx4_product(c, s[:, :8], c, s)
    with pytest.raises(ValueError, match="columns"):
        difr.mx4_dequantize(c, s, 385)
    with pytest.raises(ValueError, match="columns"):
        difr.mx4_dequantize(c, s, 256)
    with pytest.raises(ValueError, match="out must be"):
        difr.mx4_product(c, s, c, s, out=torch.zeros(5, 6, device=DEV, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="out must be"):
        difr.mx4_product(c, s, c, s, out=torch.zeros(5, 5, device=DEV))
    with pytest.raises(ValueError, match="x must be"):
        difr.mx4_quantize(torch.ones(5, 300, device=DEV).half())


def test_a_4_bit_head_under_the_scores_and_a_policy_step(difr):
    """A server runs its head in 4 bits: the verifier forms the same logits, finds the server's tokens in them, and the rollout is
    trained on."""
    g = torch.Generator().manual_seed(3)
    N, V, d, S = 48, 3001, 500, 3
    hidden, weight = torch.randn(N, d, generator=g), torch.randn(V, d, generator=g) / math.sqrt(d) * 3
    h, w = difr.mx4_quantize(hidden.bfloat16().to(DEV)), difr.mx4_quantize(weight.bfloat16().to(DEV))
    logits = difr.mx4_product(h["codes"], h["scales"], w["codes"], w["scales"])
    seeds = torch.arange(1, S + 1, dtype=torch.int64, device=DEV)
    sid = torch.arange(N, dtype=torch.int32, device=DEV) // (N // S)
    pos = torch.arange(N, dtype=torch.int32, device=DEV) % (N // S)
    at = (logits, 1.0, seeds, sid, pos)
    tokens = difr.gumbel_score(*at, None)["argmax"]
    honest, _ = difr.score_both(*at, tokens, tokens)
    assert honest["margin"].eq(0).all()
    x = logits.cpu()
    logp, H, lp = ref.rows(x, 1.0, tokens.cpu())
    o = difr.token_logprob(logits, 1.0, tokens)
    ref.assert_within(o["logp"], logp, ref.logp_bound(lp, logp))
    A = torch.randn(N, generator=g)
    p = difr.policy_loss(logits, 1.0, tokens, A.to(DEV), old_logp=o["logp"])
    want = ref.gradient(lp, H, tokens.cpu(), 1.0, -A.double() / N)
    ref.assert_within(p["grad"], want, ref.grad_bound(want, lp, H, 1.0, A / N, None, torch.bfloat16) + 1e-5 * want.abs())
    off = torch.tensor([0, 16, 32, 48, 48], dtype=torch.int64, device=DEV)
    q = difr.preference_loss(logits, 1.0, tokens, off, 0.1)
    total = torch.stack([logp[0:16].sum(), logp[16:32].sum(), logp[32:48].sum(), torch.zeros(()).double()])
    ref.assert_within(q["seq_logp"], total, 1e-6 * total.abs())


def test_the_head_is_captured_and_replayed(difr):
    w = difr.mx4_quantize((torch.randn(1500, 640, generator=torch.Generator().manual_seed(1)) / 25).to(DEV))
    for N in (5, 200):
        x = torch.zeros(N, 640, dtype=torch.bfloat16, device=DEV)

        def step():
            q = difr.mx4_quantize(x)
            return difr.mx4_product(q["codes"], q["scales"], w["codes"], w["scales"]), difr.mx4_dequantize(q["codes"], q["scales"], 640)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = step()
        for seed in (1, 2, 3):
            x.copy_(torch.randn(N, 640, generator=torch.Generator().manual_seed(seed)))
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in captured]
            eager = step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, eager)), (N, seed)
