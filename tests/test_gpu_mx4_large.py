"""The 4-bit product where a workgroup has more than one tile: large heads under few rows (with and without reads past the caches), batches of
more tiles than compute units, and scales at their ends in the batch kernel."""
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


def _rows(difr, seed, N, d, scale):
    """Quantised rows of different size, and their values in 64 bits."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(N, d, generator=g, device=DEV) * (scale * torch.randn(N, 1, generator=g, device=DEV)).exp()
    q = difr.mx4_quantize(x)
    return (q["codes"], q["scales"]), difr.mx4_dequantize(q["codes"], q["scales"], d, dtype=torch.float32)


def _check(difr, a, va, b, vb, dtype):
    """Products of 4-bit values are exact in fp32, and a sum of K of them is off by at most K half steps of the sum of magnitudes,
    whatever its order; the result is rounded once.  Nothing beside the output is written."""
    N, V, K = va.shape[0], vb.shape[0], va.shape[1]
    buf = torch.full((N + 1, V + 5), 7.0, dtype=dtype, device=DEV)
    got = buf[:N, 3:V + 3]
    difr.mx4_product(*a, *b, dtype=dtype, out=got)
    assert buf[N].eq(7).all() and buf[:, :3].eq(7).all() and buf[:, V + 3:].eq(7).all(), "what lies around it"
    x = va.double()
    for v in range(0, V, 16384):
        w = vb[v:v + 16384].double().t().contiguous()
        want, size = x @ w, x.abs() @ w.abs()
        off = (got[:, v:v + 16384].double() - want).abs() - ref.EPS[dtype] * want.abs() - 2.0 ** -24 * K * size
        assert off.max() <= 0, (v, float(off.max()))
    again = difr.mx4_product(*a, *b, dtype=dtype)
    assert torch.equal(again, got), "the same call, the same bits"


@pytest.mark.parametrize("V,d", [(65473, 384), (65505, 512), (70001, 384), (131111, 130)])
def test_few_rows_by_a_large_head(difr, V, d):
    b, vb = _rows(difr, V, V, d, 0.5)
    for N in (1, 32, 33, 64, 65, 128):
        a, va = _rows(difr, N, N, d, 2.0)
        for dtype in (torch.bfloat16, torch.float32):
            _check(difr, a, va, b, vb, dtype)


@pytest.mark.parametrize("V,d", [(151937, 4096), (140001, 3968)])
def test_few_rows_by_a_head_that_is_read_past_the_caches(difr, V, d):
    b, vb = _rows(difr, V, V, d, 0.5)
    assert b[0].numel() > 256 << 20
    for N, dtype in ((1, torch.bfloat16), (17, torch.float32), (50, torch.bfloat16), (128, torch.float32), (100, torch.bfloat16)):
        a, va = _rows(difr, N, N, d, 2.0)
        _check(difr, a, va, b, vb, dtype)


@pytest.mark.parametrize("N,V,d", [(300, 151937, 640), (1100, 20003, 512), (1025, 33000, 384), (129, 151936, 128), (2000, 40007, 130)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_batches_of_more_tiles_than_compute_units(difr, N, V, d, dtype):
    b, vb = _rows(difr, V, V, d, 0.5)
    a, va = _rows(difr, N, N, d, 2.0)
    _check(difr, a, va, b, vb, dtype)


@pytest.mark.parametrize("N", [20, 60, 120, 200, 530])
@pytest.mark.parametrize("d", [256, 384])
def test_extreme_scales_and_nan(difr, N, d):
    V = 700
    a, b = torch.ones(N, d), torch.ones(V, d)
    a[1] *= 2.0 ** 100
    a[2] *= 2.0 ** -126
    b[1] *= 2.0 ** -100
    b[2] *= 2.0 ** 20
    a[3, 40], b[3, 200], a[N - 1, d - 1], b[V - 1, 31] = math.nan, math.inf, math.inf, math.nan
    a[4, :128], b[4, 128:] = 0, 0
    a[5, 32:64] *= 2.0 ** 90
    b[600, 32:64] *= 2.0 ** -90
    va, vb = ref.mx4(a)[2], ref.mx4(b)[2]
    qa, qb = difr.mx4_quantize(a.to(DEV)), difr.mx4_quantize(b.to(DEV))
    got = difr.mx4_product(qa["codes"], qa["scales"], qb["codes"], qb["scales"], dtype=torch.float32)
    want = va @ vb.t()
    # (2^-126 2^-100 256 = 2^-218 has no place in fp32: what is below its smallest normal number, 2^-126, may come out as 0)
    ref.assert_within(got, want, 2.0 ** -24 * d * (va.abs().nan_to_num(0) @ vb.abs().nan_to_num(0).t()) + 2.0 ** -126, "product")
