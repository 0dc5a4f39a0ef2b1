"""4-bit integers with group scales against their definition: codes, values, and products of a few hidden states."""
import math

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


def _same(a, b):
    return torch.equal(a.cpu().double().nan_to_num(nan=-77.0), b.double().nan_to_num(nan=-77.0))


def _rows(t, offset, gap, fill=math.nan):
    """The tensor on the device as a view whose rows start anywhere; what lies between them is `fill`."""
    N, d = t.shape
    buf = torch.full((offset + N * (d + gap),), fill, dtype=t.dtype, device=DEV)
    view = buf[offset:].view(N, d + gap)[:, :d]
    view.copy_(t)
    return view


@pytest.mark.parametrize("N,d", [(1, 1), (3, 31), (2, 32), (5, 63), (4, 128), (2, 129), (7, 1000), (33, 4096)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group,zero_points,offset,gap", [(32, True, 0, 0), (64, False, 1, 0), (128, True, 5, 3), (128, False, 0, 0), (64, True, 2, 1)])
def test_quantize_and_back(difr, N, d, dtype, group, zero_points, offset, gap):
    g = torch.Generator().manual_seed(N * 100 + d)
    x = (torch.randn(N, d, generator=g) * (2 * torch.randn(N, 1, generator=g)).exp() + 0.3).to(dtype)
    codes, scales, zeros, values = ref.int4(x, group, zero_points)
    q = difr.int4_quantize(_rows(x, offset, gap), group=group, zero_points=zero_points)
    assert torch.equal(q["codes"].cpu(), codes) and torch.equal(q["scales"].cpu().view(torch.int16), scales.view(torch.int16))
    assert ("zeros" in q) == zero_points and (not zero_points or torch.equal(q["zeros"].cpu(), zeros))
    assert _same(difr.int4_dequantize(q["codes"], q["scales"], d, q.get("zeros"), dtype=torch.float32), values[:, :d])
    assert _same(difr.int4_dequantize(q["codes"], q["scales"], d, q.get("zeros")), values[:, :d].to(torch.bfloat16))


@pytest.mark.parametrize("zero_points", [False, True])
def test_groups_that_are_special(difr, zero_points):
    half = torch.arange(-16, 16).float()
    rows = [half / 2, half / 2 + 0.25, torch.zeros(32), -torch.zeros(32), half.abs(), -half.abs(), half * 2.0 ** -120, half * 2.0 ** -140,
            half * 2.0 ** 120, torch.full((32,), 3.0), torch.full((32,), -3.0), torch.full((32,), 3e38)]
    for bad in (math.nan, math.inf, -math.inf):
        r = half.clone()
        r[5] = bad
        rows.append(r)
    huge = torch.full((32,), 3e38)
    huge[::2] = -3e38                                   # a difference beyond fp32
    rows.append(huge)
    x = torch.stack(rows)
    x = torch.cat([x, x.flip(0), x, x], 1)
    codes, scales, zeros, values = ref.int4(x, 32, zero_points)
    q = difr.int4_quantize(x.to(DEV), group=32, zero_points=zero_points)
    good = ~scales.isnan()
    assert torch.equal(q["scales"].cpu().isnan(), ~good)
    assert torch.equal(q["scales"].cpu()[good], scales[good])
    back = difr.int4_dequantize(q["codes"], q["scales"], 128, q.get("zeros"), dtype=torch.float32).cpu()
    assert _same(back, values.float().double())


def _matrix(difr, V, d, group, zero_points, seed, scale_of=None):
    """Random codes (padding too), scales and zero points, and the values [V, d] in 64 bits."""
    g = torch.Generator().manual_seed(seed)
    K = difr.int4_padded(d)
    c = torch.randint(0, 16, (V, K), generator=g, dtype=torch.uint8)
    s = (scale_of(g, V, K // group) if scale_of else torch.rand(V, K // group, generator=g) + 0.1).to(torch.bfloat16)
    z = torch.randint(0, 16, (V, K // group), generator=g, dtype=torch.uint8) if zero_points else None
    w = c.double() - (8.0 if z is None else z.double().repeat_interleave(group, 1))
    w = w * s.double().repeat_interleave(group, 1)
    return (c[:, 0::2] | (c[:, 1::2] << 4)).to(DEV), s.to(DEV), None if z is None else z.to(DEV), w[:, :d]


SHAPES = [(1, 1, 1), (1, 16, 128), (2, 17, 31), (3, 64, 256), (5, 100, 129), (15, 1000, 1000), (16, 33, 4096), (17, 250, 2000), (31, 129, 512), (20, 9001, 700),
          (33, 1024, 640), (48, 77, 384), (64, 500, 4096), (65, 96, 1024), (130, 40, 896), (16, 70000, 300), (3, 35000, 5000), (40, 40000, 260), (70, 20000, 130),
          (1100, 33, 200)]


@pytest.mark.parametrize("N,V,d", SHAPES)
@pytest.mark.parametrize("group,zero_points", [(32, True), (64, False), (128, True), (128, False)])
@pytest.mark.parametrize("hidden,out", [(torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
def test_whole_numbers_are_exact(difr, N, V, d, group, zero_points, hidden, out):
    """Hidden states of small whole numbers and scales of 1, 2 and 4: every partial sum, with the codes' offsets of up to 32, is a whole
    number below 2^24 (4096 elements * 32 * 4 * 8 = 2^22), so the only rounding is the last."""
    codes, scales, zeros, w = _matrix(difr, V, d, group, zero_points, V + d, lambda g, r, c: 2.0 ** torch.randint(0, 3, (r, c), generator=g))
    h = torch.randint(-8, 9, (N, d), generator=torch.Generator().manual_seed(N)).to(hidden)
    want = (h.double() @ w.t()).to(out)
    got = difr.int4_product(_rows(h, 3, 5), codes, scales, zeros, dtype=out)
    assert got.dtype == out and torch.equal(got.cpu(), want)


@pytest.mark.parametrize("N,V,d", [s for s in SHAPES if s[2] > 100])
@pytest.mark.parametrize("group,zero_points", [(32, False), (64, True), (128, True)])
@pytest.mark.parametrize("hidden", [torch.bfloat16, torch.float32])
def test_product(difr, N, V, d, group, zero_points, hidden):
    codes, scales, zeros, w = _matrix(difr, V, d, group, zero_points, V + d)
    h = (torch.randn(N, d, generator=torch.Generator().manual_seed(N)) * 3).to(hidden)
    want = h.double() @ w.t()
    # a running sum of `group` products of an element by a code offset by up to 32, scaled, summed over the groups: each of at most
    # group + d / group + 8 additions is off by 2^-23 (the matrix cores may cut) of what has been added up
    size = h.double().abs() @ (w.abs() + 32 * scales.cpu().double().repeat_interleave(group, 1)[:, :d]).t()
    bound = size * (group + difr.int4_padded(d) // group + 8) * 2.0 ** -23
    got = difr.int4_product(h.to(DEV), codes, scales, zeros, dtype=torch.float32)
    assert ((got.cpu().double() - want).abs() <= bound + want.abs() * 2.0 ** -24).all()
    # what the bound does not see: on the whole the sums are as good as fp32 sums are
    error = (got.cpu().double() - want).square().mean().sqrt() / want.square().mean().sqrt()
    assert error < 2.0 ** -19, error
    half = difr.int4_product(h.to(DEV), codes, scales, zeros)
    assert ((half.cpu().double() - want).abs() <= bound + (want.abs() + bound) * 2.0 ** -8).all()


def test_out_with_a_pitch_and_what_lies_beside_it(difr):
    codes, scales, zeros, w = _matrix(difr, 333, 256, 64, True, 5)
    h = torch.randint(-4, 5, (20, 256)).to(torch.bfloat16)
    buf = torch.full((20, 340), 7.0, device=DEV)
    h_dev = h.to(DEV)
    v0 = buf._version
    got = difr.int4_product(h_dev, codes, scales, zeros, dtype=torch.float32, out=buf[:, 3:336])
    assert got.data_ptr() == buf[:, 3:].data_ptr() and buf._version > v0
    assert torch.equal(buf[:, 3:336].cpu(), difr.int4_product(h_dev, codes, scales, zeros, dtype=torch.float32).cpu())
    assert buf[:, :3].eq(7).all() and buf[:, 336:].eq(7).all()


def test_rows_do_not_touch_each_other(difr):
    """A row's logits are the same alone and among others, and what is no number stays in its row."""
    codes, scales, zeros, w = _matrix(difr, 500, 1000, 128, True, 6)
    h = torch.randn(64, 1000, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    whole = difr.int4_product(h.to(DEV), codes, scales, zeros, dtype=torch.float32)
    for n in (1, 2, 16, 17, 40):
        assert torch.equal(difr.int4_product(h[:n].to(DEV), codes, scales, zeros, dtype=torch.float32), whole[:n]), n
    h[3, 7], h[20, 999], h[41, 0] = math.nan, math.inf, -math.inf
    got = difr.int4_product(h.to(DEV), codes, scales, zeros, dtype=torch.float32)
    bad = torch.zeros(64, dtype=torch.bool)
    bad[[3, 20, 41]] = True
    assert torch.equal(got[~bad], whole[~bad]) and not got[bad].isfinite().any()


@pytest.mark.parametrize("V,d,group", [(17000, 640, 64), (20011, 2100, 128), (16500, 300, 32)])
@pytest.mark.parametrize("hidden", [torch.bfloat16, torch.float32])
def test_a_row_alone_and_among_others(difr, V, d, group, hidden):
    """Large heads: the same bits however many rows there are, from whatever stream and into whatever tensor."""
    codes, scales, zeros, _ = _matrix(difr, V, d, group, True, 7)
    h = torch.randn(100, d, generator=torch.Generator().manual_seed(2)).to(hidden).to(DEV)
    whole = difr.int4_product(h, codes, scales, zeros, dtype=torch.float32)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for n in (1, 5, 16, 17, 33, 49, 65):
        with torch.cuda.stream(stream):
            got = difr.int4_product(h[100 - n:], codes, scales, zeros, dtype=torch.float32)
        torch.cuda.synchronize()
        assert torch.equal(got, whole[100 - n:]), n


def test_empty(difr):
    codes, scales, zeros, w = _matrix(difr, 5, 128, 128, False, 1)
    assert difr.int4_product(torch.zeros(0, 128, dtype=torch.bfloat16, device=DEV), codes, scales).shape == (0, 5)
    assert difr.int4_product(torch.zeros(3, 128, dtype=torch.bfloat16, device=DEV), codes[:0], scales[:0]).shape == (3, 0)
    assert difr.int4_quantize(torch.zeros(0, 5, device=DEV))["codes"].shape == (0, 64)


def test_a_quantised_head_gives_the_dense_products(difr):
    g = torch.Generator().manual_seed(9)
    w = (torch.randn(700, 2048, generator=g) / 45).to(torch.bfloat16).to(DEV)
    h = torch.randn(6, 2048, generator=g).to(torch.bfloat16).to(DEV)
    q = difr.int4_quantize(w, group=64, zero_points=True)
    dense = difr.int4_dequantize(q["codes"], q["scales"], 2048, q["zeros"], dtype=torch.float32)
    assert (dense - w.float()).abs().max() < 0.02       # half a step of a sixteenth of a group's range
    want = h.double().cpu() @ dense.double().cpu().t()
    got = difr.int4_product(h, q["codes"], q["scales"], q["zeros"], dtype=torch.float32)
    assert (got.cpu().double() - want).abs().max() < 1e-4 * want.abs().max()


def _bound(h, w, group):
    """Of fp32 accumulation: group + d / group + 8 additions, each off by up to 2^-23 (the matrix cores may cut) of what has been added up, and
    states cut below 2^-39 of their row's largest: its scale is a power of two that brings it to 2^15 at least, and fp16 numbers end at 2^-24."""
    h, size = h.double().abs(), h.double().abs() @ w.abs().t()
    return size * (group + w.shape[1] // group + 9) * 2.0 ** -23 + h.amax(1, keepdim=True) * w.abs().sum(1) * 2.0 ** -39


SOME = [(1, 3, 300, 8), (1, 100, 256, 128), (7, 17000, 300, 64), (16, 500, 1000, 32), (17, 300, 1030, 128), (33, 17000, 200, 32), (50, 17000, 130, 64), (64, 16500, 256, 128)]


@pytest.mark.parametrize("N,V,d,group", [(n, v, d, max(g, 32)) for n, v, d, g in SOME])
@pytest.mark.parametrize("zero_points", [False, True])
@pytest.mark.parametrize("hidden", [torch.bfloat16, torch.float32])
def test_codes_at_their_zero_points_add_nothing(difr, N, V, d, group, zero_points, hidden):
    """Whatever the states: elements whose code is the zero point have the value 0.  All of them so: the sum is 0.  Those of channels that are much larger
    than the others: what is lost of the others does not depend on them, beyond 2^-39."""
    g = torch.Generator().manual_seed(N + V)
    codes, scales, zeros, _ = _matrix(difr, V, d, group, zero_points, d)
    K = difr.int4_padded(d)
    z = (torch.full((V, K // group), 8, dtype=torch.uint8) if zeros is None else zeros.cpu()).repeat_interleave(group, 1)
    h = (torch.randn(N, d, generator=g) * (4 * torch.randn(N, d, generator=g)).exp()).to(hidden)
    none = (z[:, 0::2] | (z[:, 1::2] << 4)).to(DEV)
    assert difr.int4_product(h.to(DEV), none, scales, zeros, dtype=torch.float32).eq(0).all()
    c = torch.randint(0, 16, (V, K), generator=g, dtype=torch.uint8)
    h = torch.randn(N, d, generator=g)
    for k, times in ((5, 2.0 ** 13), (d // 2, -2.0 ** 10), (d - 1, 2.0 ** 16)):
        h[:, k] = times * (1 + torch.rand(N, generator=g))
        c[:, k] = z[:, k]
    h = h.to(hidden)
    w = ((c.double() - z.double()) * scales.cpu().double().repeat_interleave(group, 1))[:, :d]
    got = difr.int4_product(h.to(DEV), (c[:, 0::2] | (c[:, 1::2] << 4)).to(DEV), scales, zeros, dtype=torch.float32)
    assert ((got.cpu().double() - h.double() @ w.t()).abs() <= _bound(h, w, group)).all()


@pytest.mark.parametrize("N,V,d,group", [(n, v, d, max(g, 32)) for n, v, d, g in SOME])
@pytest.mark.parametrize("hidden", [torch.bfloat16, torch.float32])
def test_states_of_every_size(difr, N, V, d, group, hidden):
    """Rows near the ends of fp32, of one sign and of both, and rows whose elements differ by 2^30: as good as others."""
    g = torch.Generator().manual_seed(N)
    codes, scales, zeros, w = _matrix(difr, V, d, group, True, 3, lambda g, r, c: (torch.rand(r, c, generator=g) + 0.5) * 2.0 ** -12)
    sizes = (2.0 ** 127, 2.0 ** 117, 1.0, 2.0 ** -60, 2.0 ** -110)
    for first in range(0, len(sizes), N):
        u = torch.rand(N, d, generator=g, dtype=torch.float64)
        h = torch.stack([(u[n] + 0.25 if n % 2 else u[n] - 0.5) * sizes[(first + n) % len(sizes)] for n in range(N)])
        h[:, ::7] *= 2.0 ** -30
        h = h.to(hidden)
        assert h.isfinite().all()
        want = h.double() @ w.t()
        want[want.abs() > torch.finfo(torch.float32).max] = math.nan                    # (infinities are right too)
        got = difr.int4_product(h.to(DEV), codes, scales, zeros, dtype=torch.float32).cpu().double()
        near = want.abs() > 2.0 ** 127
        good = ((got - want).abs() <= _bound(h, w, group) + 2.0 ** -149) | want.isnan() | (near & ~got.isfinite())
        assert good.all()


@pytest.mark.parametrize("N,V,d,group", [(1, 1024, 256, 128), (9, 17000, 512, 128), (40, 2000, 640, 128)])
@pytest.mark.parametrize("zero_points", [False, True])
def test_fp32_states_are_summed_in_fp32(difr, N, V, d, group, zero_points):
    """Normal weights, most of whose codes are near their zero points.  What the bound over all signs does not see: independent errors add as squares.  n = 2 (3 d / 32 + d / group) accumulations (a matrix instruction
    for each part of 32 states, taken to round twice) of at most 2^-23 of the sum: sqrt(n) 2^-23 of it altogether."""
    weights = torch.randn(V, d, generator=torch.Generator().manual_seed(11))
    codes, scales, zeros, w = ref.int4(weights, group, zero_points)
    codes, scales, zeros, w = codes.to(DEV), scales.to(DEV), None if zeros is None else zeros.to(DEV), w[:, :d]
    h = torch.randn(N, d, generator=torch.Generator().manual_seed(4))
    want = h.double() @ w.t()
    got = difr.int4_product(h.to(DEV), codes, scales, zeros, dtype=torch.float32).cpu().double()
    error = (got - want).square().mean().sqrt() / want.square().mean().sqrt()
    assert error < math.sqrt(2 * (3 * d // 32 + d // group)) * 2.0 ** -23, float(error)


@pytest.mark.parametrize("N,V,d,group", [(1, 100, 256, 128), (5, 17000, 300, 64), (33, 500, 1000, 32), (20, 17000, 130, 128)])
@pytest.mark.parametrize("hidden", [torch.bfloat16, torch.float32])
def test_small_states_beside_a_large_one(difr, N, V, d, group, hidden):
    """A channel of 1 whose codes are the zero points, and others of up to 8 times 2^-31 (in fp16, scaled, numbers below the normal ones): exact, with
    scales of 1, 2 and 4, as the sums are whole numbers below 2^24 times 2^-31."""
    g = torch.Generator().manual_seed(V + d)
    codes, scales, zeros, _ = _matrix(difr, V, d, group, True, 9, lambda g, r, c: 2.0 ** torch.randint(0, 3, (r, c), generator=g))
    K = difr.int4_padded(d)
    z = zeros.cpu().repeat_interleave(group, 1)
    c = torch.randint(0, 16, (V, K), generator=g, dtype=torch.uint8)
    c[:, 7] = z[:, 7]
    h = torch.randint(-8, 9, (N, d), generator=g) * 2.0 ** -31
    h[:, 7] = 1.0
    w = ((c.double() - z.double()) * scales.cpu().double().repeat_interleave(group, 1))[:, :d]
    got = difr.int4_product(h.to(hidden).to(DEV), (c[:, 0::2] | (c[:, 1::2] << 4)).to(DEV), scales, zeros, dtype=torch.float32)
    assert torch.equal(got.cpu().double(), h.double() @ w.t())


@pytest.mark.parametrize("d", [1, 4, 7])
@pytest.mark.parametrize("hidden", [torch.bfloat16, torch.float32])
def test_short_states_of_every_size(difr, d, hidden):
    """Fewer than eight elements, near the ends of fp32: d products and additions, each rounded once."""
    codes, scales, zeros, w = _matrix(difr, 300, d, 32, True, 3, lambda g, r, c: (torch.rand(r, c, generator=g) + 0.5) * 2.0 ** -12)
    h = (torch.rand(6, d, generator=torch.Generator().manual_seed(1), dtype=torch.float64) + 0.5) * torch.tensor([2.0 ** 127, -2.0 ** 126, 2.0 ** 120, 1.0, 2.0 ** -60, 2.0 ** -100])[:, None]
    h = h.clamp(-3e38, 3e38).to(hidden)
    got = difr.int4_product(h.to(DEV), codes, scales, zeros, dtype=torch.float32).cpu().double()
    assert ((got - h.double() @ w.t()).abs() <= (h.double().abs() @ w.abs().t()) * d * 2.0 ** -24).all()


@pytest.mark.parametrize("N,V,d", [(17, 100, 8), (33, 17000, 9), (40, 50, 100), (20, 17000, 127), (3, 100, 20000), (2, 17000, 8200), (17, 100, 8200), (20, 40, 20001), (7, 17000, 2049)])
@pytest.mark.parametrize("group,zero_points", [(32, True), (64, True), (128, False)])
@pytest.mark.parametrize("hidden", [torch.bfloat16, torch.float32])
def test_short_and_long_states_are_exact(difr, N, V, d, group, zero_points, hidden):
    """Half a slab and less, rows that end anywhere in it, and more elements than are kept while a row's largest is sought: whole numbers below
    2^24 (20,001 elements * 15 * 4 * 8), so that nothing is rounded."""
    codes, scales, zeros, w = _matrix(difr, V, d, group, zero_points, V + d, lambda g, r, c: 2.0 ** torch.randint(0, 3, (r, c), generator=g))
    h = torch.randint(-8, 9, (N, d), generator=torch.Generator().manual_seed(N)).to(hidden)
    h[0, d - 1], h[N - 1, 0] = 8, -8
    got = difr.int4_product(_rows(h, 1, 3), codes, scales, zeros, dtype=torch.float32)
    assert torch.equal(got.cpu().double(), h.double() @ w.t())


@pytest.mark.parametrize("N", [3, 20, 70])
@pytest.mark.parametrize("hidden", [torch.bfloat16, torch.float32])
def test_products_captured_and_replayed(difr, N, hidden):
    """Two graphs of one shape, replayed in turn with states of other sizes and eager calls between them."""
    codes, scales, zeros, _ = _matrix(difr, 700, 640, 64, True, 5)
    h = [torch.empty(N, 640, dtype=hidden, device=DEV) for _ in range(2)]
    g = torch.Generator().manual_seed(8)
    load = lambda size: [t.copy_(torch.randn(N, 640, generator=g) * size) for t in h]
    step = lambda t: difr.int4_product(t, codes, scales, zeros, dtype=torch.float32)
    load(1.0)
    step(h[0])
    torch.cuda.synchronize()
    graphs, got = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for graph, t in zip(graphs, h):
        with torch.cuda.graph(graph):
            got.append(step(t))
    for size in (1.0, 1e-20, 1e20, 3.0):
        load(size)
        want = [step(t) for t in h]
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and not torch.equal(got[0], got[1])
