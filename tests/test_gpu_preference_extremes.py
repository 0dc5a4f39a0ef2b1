"""The preference loss where a reply holds a token that the policy cannot give: the log ratio is infinite, the loss is what the limit says."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = math.inf


@pytest.fixture(scope="module")
def difr():
    import paper_2511_02620_amd as m
    m.load_library()
    return m


@pytest.mark.parametrize("eps", [0.0, 0.1, 1.0])
@pytest.mark.parametrize("V", [64, 100003])
def test_a_token_without_probability(difr, eps, V):
    """Pairs: masked token in the rejected reply (h = inf), in the chosen one (h = -inf), in neither, and in both."""
    g = torch.Generator().manual_seed(V)
    x = torch.randn(16, V, generator=g)
    tok = torch.randint(0, V, (16,), generator=g, dtype=torch.int32)
    for n in (3, 4, 13, 14):
        x[n, tok[n]] = -INF
    off = torch.arange(0, 17, 2, dtype=torch.int64, device=DEV)
    xd, td = x.to(DEV), tok.to(DEV)
    w = torch.tensor([0.5, 0.25, 1.0, 0.0], device=DEV)
    o = difr.preference_loss(xd, 1.0, td, off, 0.5, pair_weights=w, label_smoothing=eps)
    assert o["seq_logp"].isinf().tolist() == [n in (1, 2, 6, 7) for n in range(8)]
    h = 0.5 * (o["seq_logp"].double()[4] - o["seq_logp"].double()[5]).item()
    mid = (1 - eps) * math.log1p(math.exp(-h)) + eps * math.log1p(math.exp(h))
    first, second = (0.0 if eps == 0 else INF), (0.0 if eps == 1 else INF)
    got = o["pair_loss"].tolist()
    assert got[:2] == [first, second] and abs(got[2] - mid) < 1e-6 * (1 + abs(mid)) and math.isnan(got[3])
    want = mid + (0.5 * first if eps == 0 else INF) + (0.25 * second if eps == 1 else INF)
    assert o["loss"].item() == want or abs(o["loss"].item() - want) < 1e-6 * (1 + abs(mid))
    # sigma(inf) = 1: what flows back is a number everywhere, and nothing where the weight is 0
    a = o["grad_logp"]
    assert a[:4].tolist() == pytest.approx([0.25 * eps] * 2 + [-0.25 * eps] * 2, abs=1e-8)
    assert a[4:8].tolist() == pytest.approx([-0.125 * (1 - eps)] * 2 + [0.125 * (1 - eps)] * 2, abs=1e-8)
    assert a[12:].eq(0).all() and o["grad"][12:].eq(0).all() and torch.isfinite(o["grad"]).all()
