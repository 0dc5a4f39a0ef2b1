"""Calls on logged tokens and 4-bit rows with something else in a tensor's place, or with an output that nothing is written to."""
import pytest
import torch

import paper_2511_02620_amd as difr


@pytest.mark.parametrize("bad", [None, 3, [1.0]])
def test_what_is_no_tensor_is_named(bad):
    c = torch.zeros(4, 64, dtype=torch.uint8)
    t, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    for call, name in ((lambda: difr.token_logprob(bad, 1.0, t), "logits"), (lambda: difr.policy_loss(bad, 1.0, t, f), "logits"),
                       (lambda: difr.mx4_quantize(bad), "x"), (lambda: difr.mx4_dequantize(bad, c, 128), "codes"),
                       (lambda: difr.mx4_dequantize(c, bad, 128), "scales"), (lambda: difr.mx4_product(bad, c, c, c), "a_codes")):
        with pytest.raises(ValueError, match="%s must be a tensor" % name):
            call()


@pytest.mark.gpu
def test_on_the_device():
    dev = "cuda:0"
    x, t, f = torch.zeros(4, 8, device=dev), torch.zeros(4, dtype=torch.int32, device=dev), torch.zeros(4, device=dev)
    off, out = torch.tensor([0, 2, 4], device=dev), torch.full((4, 8), 7.0, device=dev)
    q = difr.mx4_quantize(x)
    for call, message in ((lambda: difr.token_logprob_backward(x, 1.0, t, None, f), "stats must be a tensor"),
                          (lambda: difr.token_logprob_backward(x, 1.0, t, torch.zeros(4, 2, device=dev), None), "grad_logp must be a tensor"),
                          (lambda: difr.preference_loss(x, 1.0, t, None, 0.1), "seq_offsets must be a tensor"),
                          (lambda: difr.policy_loss(x, 1.0, t, f, out=3), "out must be a tensor"),
                          (lambda: difr.policy_loss(x, 1.0, t, f, want_grad=False, out=out), "want_grad"),
                          (lambda: difr.preference_loss(x, 1.0, t, off, 0.1, want_grad=False, out=out), "want_grad"),
                          (lambda: difr.mx4_product(q["codes"], q["scales"], q["codes"], None), "b_scales must be a tensor")):
        with pytest.raises(ValueError, match=message):
            call()
    assert out.eq(7).all()
    codes = torch.zeros(4 * 64 + 8, dtype=torch.uint8, device=dev)[8:].view(4, 64)
    with pytest.raises(difr.DifrError, match="not aligned"):
        difr.mx4_dequantize(codes, q["scales"], 8)
