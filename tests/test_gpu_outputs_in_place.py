"""Tensors of the caller's that a call writes to: a graph that has saved one finds out."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def difr():
    import paper_2511_02620_amd as m
    m.load_library()
    return m


def _calls(difr, x, t, A):
    off = torch.tensor([0, 2, 4], device=DEV)
    stats = difr.token_logprob(x.detach(), 1.0, t)["stats"]
    return {"policy": lambda T, out: difr.policy_loss(x, T, t, A, out=out),
            "preference": lambda T, out: difr.preference_loss(x, T, t, off, 0.1, out=out),
            "backward": lambda T, out: difr.token_logprob_backward(x, T, t, stats, A, out=out)}


@pytest.mark.parametrize("which", ["policy", "preference", "backward"])
def test_a_graph_that_saved_the_logits_refuses_its_backward_pass(difr, which):
    w = torch.randn(4, 40, device=DEV, requires_grad=True)
    t, A = torch.zeros(4, dtype=torch.int32, device=DEV), torch.ones(4, device=DEV)
    x = w * 2.0
    z = (x * x).sum()                                   # saves x
    call = _calls(difr, x, t, A)[which]
    version = x._version
    other = torch.empty(4, 40, device=DEV)
    call(1.0, other)
    assert x._version == version and other._version == 1
    with pytest.raises(difr.DifrError):
        call(0.0, x)
    assert x._version == version, "nothing has been written"
    call(1.0, x)
    assert x._version == version + 1
    with pytest.raises(RuntimeError, match="inplace operation"):
        z.backward()
    # logits that no graph has saved: their place takes the gradient, which goes on from there
    y = w * 2.0
    _calls(difr, y, t, A)[which](1.0, y)
    g = y.detach().clone()
    y.backward(y.detach())
    assert torch.equal(w.grad, 2.0 * g)


def test_inference_tensors_are_written(difr):
    with torch.inference_mode():
        x = torch.randn(4, 40, device=DEV)
        t, A = torch.zeros(4, dtype=torch.int32, device=DEV), torch.ones(4, device=DEV)
        want = difr.policy_loss(x, 1.0, t, A)["grad"]
        difr.policy_loss(x, 1.0, t, A, out=x)
    assert torch.equal(x, want)
    difr.token_logprob_backward(x, 1.0, t, torch.ones(4, 2, device=DEV), A, out=x)


def test_the_product_s_output(difr):
    q = difr.mx4_quantize(torch.randn(5, 300, device=DEV) / math.sqrt(300))
    out = torch.zeros(5, 5, dtype=torch.bfloat16, device=DEV)
    difr.mx4_product(q["codes"], q["scales"], q["codes"], q["scales"], out=out)
    assert out._version == 1
