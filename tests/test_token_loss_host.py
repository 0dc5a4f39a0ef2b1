"""What the calls on logged tokens and on 4-bit rows refuse before they touch the device, and the plain forms against autograd."""
import ctypes as C

import pytest
import torch

import paper_2511_02620_amd as difr
import token_loss_ref as ref
from paper_2511_02620_amd import binding

OK, NULL, SHAPE, DTYPE, TEMP, ALIGN, _, _, ARG = range(9)
FAKE = 0x1000                                        # never dereferenced: every call below fails validation first


def _rows(**kw):
    r = binding._TokenRows(FAKE, 0, 4, 16, 16, 1.0, None, FAKE)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _policy(**kw):
    p = binding._Policy(FAKE, FAKE, FAKE, FAKE, 0.2, 0.2, 0.1, 0.0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _pref(**kw):
    p = binding._Preference(FAKE, 4, None, None, None, 0.1, 0.0, 0.0, 0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _calls(lib):
    def logprob(r, logp=FAKE, flags=FAKE, ws=None, n=0):
        return lib.difr_token_logprob(C.byref(r), logp, None, None, flags, ws, n, None)

    def backward(r, stats=FAKE, ent=None, ga=FAKE, ge=None, grad=FAKE, ld=16):
        return lib.difr_token_logprob_backward(C.byref(r), stats, ent, ga, ge, grad, ld, None)

    def policy(r, p=None, loss=FAKE, each=FAKE, kl=None, flags=FAKE, grad=None, ld=16, ws=None, n=0):
        return lib.difr_policy_loss(C.byref(r), C.byref(p or _policy()), loss, each, FAKE, None, kl, flags, grad, ld, ws, n, None)

    def pref(r, p=None, loss=FAKE, pair=FAKE, stats=FAKE, flags=FAKE, grad=None, ld=16, ws=None, n=0):
        return lib.difr_preference_loss(C.byref(r), C.byref(p or _pref()), loss, pair, FAKE, FAKE, stats, FAKE, flags, grad, ld, ws, n, None)

    return logprob, backward, policy, pref


def test_rows_that_every_call_refuses():
    for call in _calls(binding.load_library()):
        for bad, want in ((dict(N=-1), SHAPE), (dict(V=0), SHAPE), (dict(ld=15), SHAPE), (dict(N=1 << 31), SHAPE),
                          (dict(V=1 << 31, ld=1 << 31), SHAPE), (dict(dtype=2), DTYPE), (dict(temperature=0.0), TEMP),
                          (dict(temperature=float("nan")), TEMP), (dict(temperature=float("inf")), TEMP), (dict(logits=None), NULL),
                          (dict(tokens=None), NULL), (dict(logits=0x1001), ALIGN), (dict(dtype=1, logits=0x1002), ALIGN)):
            assert call(_rows(**bad)) == want, (call.__name__, bad)


def test_arguments_of_each_call():
    logprob, backward, policy, pref = _calls(binding.load_library())
    nan, inf = float("nan"), float("inf")
    assert logprob(_rows(), logp=None) == NULL and logprob(_rows(), flags=None) == NULL
    assert logprob(_rows(N=0)) == OK and backward(_rows(N=0)) == OK
    for kw in (dict(stats=None), dict(ga=None), dict(grad=None), dict(ge=FAKE)):
        assert backward(_rows(), **kw) == NULL, kw
    assert backward(_rows(), ld=15) == SHAPE and backward(_rows(), grad=0x1001) == ALIGN
    for kw in (dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=nan), dict(clip_high=-1e-9), dict(clip_high=nan), dict(kl_coef=inf),
               dict(entropy_coef=nan), dict(ref_logp=None)):
        assert policy(_rows(), _policy(**kw)) == ARG, kw
    assert policy(_rows(), _policy(ref_logp=None, kl_coef=0.0), kl=FAKE) == ARG
    assert policy(_rows(), _policy(advantages=None)) == NULL
    for kw in (dict(loss=None), dict(each=None), dict(flags=None)):
        assert policy(_rows(), **kw) == NULL, kw
    assert policy(_rows(), grad=FAKE, ld=3) == SHAPE and policy(_rows(), grad=0x1001) == ALIGN
    for kw, want in ((dict(S=3), SHAPE), (dict(S=-2), SHAPE), (dict(beta=nan), ARG), (dict(margin=inf), ARG), (dict(label_smoothing=1.5), ARG),
                     (dict(label_smoothing=nan), ARG), (dict(seq_offsets=None), NULL)):
        assert pref(_rows(), _pref(**kw)) == want, kw
    for kw in (dict(loss=None), dict(pair=None), dict(flags=None), dict(stats=None, grad=FAKE)):
        assert pref(_rows(), **kw) == NULL, kw
    assert pref(_rows(), grad=FAKE, ld=15) == SHAPE and pref(_rows(), grad=0x1001) == ALIGN


def test_the_workspace_of_few_long_rows():
    lib = binding.load_library()
    logprob, _, policy, pref = _calls(lib)
    need = lib.difr_token_workspace_bytes
    assert need(0, 151936, 0) == need(-1, 151936, 0) == need(4, 0, 0) == need(4, 151936, 2) == need(4, 1000, 0) == need(65, 151936, 1) == need(1 << 31, 151936, 0) == 0
    for N in (1, 4, 64):
        for V in (100000, 151936, 1 << 24):
            for dtype in (0, 1):
                n = need(N, V, dtype)
                assert 0 < n < 1 << 20
                r = _rows(N=N, V=V, ld=V, dtype=dtype)
                for call in (logprob, policy, pref):
                    assert call(r, ws=FAKE, n=n - 1) == SHAPE
                    assert call(r, n=n) == NULL
                    assert call(r, ws=FAKE + 4, n=n) == ALIGN


def test_arguments_of_the_4_bit_calls():
    lib = binding.load_library()
    assert [difr.mx4_padded(d) for d in (-1, 0, 1, 128, 129, 4096)] == [0, 0, 128, 128, 256, 4096]
    for f in (lambda x=FAKE, t=0, N=4, d=40, ld=40, c=FAKE, s=FAKE: lib.difr_mx4_quantize(x, t, N, d, ld, c, s, None),
              lambda x=FAKE, t=0, N=4, d=40, ld=40, c=FAKE, s=FAKE: lib.difr_mx4_dequantize(c, s, N, d, x, t, ld, None)):
        for kw, want in ((dict(N=-1), SHAPE), (dict(d=0), SHAPE), (dict(ld=39), SHAPE), (dict(N=1 << 31), SHAPE),
                         (dict(d=1 << 24, ld=1 << 24), SHAPE), (dict(t=3), DTYPE), (dict(x=None), NULL), (dict(c=None), NULL),
                         (dict(s=None), NULL), (dict(x=0x1001), ALIGN), (dict(x=0x1002, t=1), ALIGN), (dict(c=0x1008), ALIGN),
                         (dict(s=0x1002), ALIGN), (dict(N=0), OK)):
            assert f(**kw) == want, kw

    def product(a=FAKE, sa=FAKE, N=4, b=FAKE, sb=FAKE, V=8, K=256, out=FAKE, t=0, ld=8, ws=FAKE, n=1 << 20):
        return lib.difr_mx4_product(a, sa, N, b, sb, V, K, out, t, ld, ws, n, None)

    for kw, want in ((dict(N=-1), SHAPE), (dict(V=-1), SHAPE), (dict(ld=7), SHAPE), (dict(K=0), SHAPE), (dict(K=64), SHAPE),
                     (dict(K=200), SHAPE), (dict(K=1 << 24), SHAPE), (dict(N=129, V=1 << 29, ld=1 << 29), SHAPE),
                     (dict(N=1 << 29), SHAPE), (dict(N=129, V=(1 << 29) - 2048, ld=1 << 29, n=1 << 40, ws=None), NULL), (dict(N=1 << 31), SHAPE), (dict(V=1 << 31, ld=1 << 31), SHAPE),
                     (dict(t=2), DTYPE), (dict(a=None), NULL), (dict(sb=None), NULL), (dict(out=None), NULL), (dict(a=0x1008), ALIGN),
                     (dict(sb=0x1002), ALIGN), (dict(out=0x1001), ALIGN), (dict(N=0), OK), (dict(V=0), OK),
                     (dict(ws=0x1008), ALIGN)):
        assert product(**kw) == want, kw
    need = lib.difr_mx4_product_workspace_bytes
    assert need(0, 8, 256) == need(4, 0, 256) == need(4, 8, 200) == need(-1, 8, 256) == 0
    big = need(4096, 5000, 640)
    assert big > 0
    assert product(N=4096, V=5000, ld=5000, K=640, n=big - 1) == SHAPE
    assert product(N=4096, V=5000, ld=5000, K=640, n=big, ws=None) == NULL


def test_host_tensors_are_refused():
    x, t, f = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    off = torch.tensor([0, 2, 4])
    for call in (lambda: difr.token_logprob(x, 1.0, t), lambda: difr.token_logprob_backward(x, 1.0, t, torch.zeros(4, 2), f),
                 lambda: difr.policy_loss(x, 1.0, t, f), lambda: difr.preference_loss(x, 1.0, t, off, 0.1)):
        with pytest.raises(ValueError, match="logits must be a GPU tensor"):
            call()
    with pytest.raises(ValueError, match="x must be"):
        difr.mx4_quantize(x)
    c = torch.zeros(4, 64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="codes must be"):
        difr.mx4_dequantize(c, c, 128)
    with pytest.raises(ValueError, match="a_codes must be"):
        difr.mx4_product(c, c, c, c)
    with pytest.raises(ValueError, match="dtype must be"):
        difr.mx4_product(c, c, c, c, dtype=torch.half)


def test_the_plain_gradient_is_autograd_s():
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(5, 9, generator=g, dtype=torch.float64) * 3).requires_grad_()
    tok, T = torch.tensor([0, 3, 8, 2, 2]), torch.tensor([0.5, 1.0, 2.0, 0.7, 1.3], dtype=torch.float64)
    a, b = torch.randn(5, generator=g, dtype=torch.float64), torch.randn(5, generator=g, dtype=torch.float64)
    lp = (x / T[:, None]).log_softmax(1)
    logp, H = lp.gather(1, tok[:, None]).squeeze(1), -(lp.exp() * lp).sum(1)
    (a * logp + b * H).sum().backward()
    rl, rh, rlp = ref.rows(x.detach(), T, tok)
    torch.testing.assert_close(rl, logp.detach(), rtol=1e-12, atol=1e-12)
    torch.testing.assert_close(rh, H.detach(), rtol=1e-12, atol=1e-12)
    torch.testing.assert_close(ref.gradient(rlp, rh, tok, T, a, b), x.grad, rtol=1e-10, atol=1e-12)


def test_the_plain_4_bit_format():
    x = torch.zeros(1, 32, dtype=torch.float64)
    x[0, :16] = torch.tensor([4.0, 5.0, 5.01, 7.9, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, -0.25, -0.75, -6.0, 0.0, -0.0])
    codes, scales, values = ref.mx4(x)
    assert values[0, :16].tolist() == [4, 4, 6, 6, 0, 0.5, 1, 1, 2, 2, 4, 0, -1, -6, 0, 0]
    assert scales.tolist() == [[127, 0, 0, 0]] and codes[0, :2].tolist() == [0x66, 0x77] and codes[0, 7].item() == 0x80
