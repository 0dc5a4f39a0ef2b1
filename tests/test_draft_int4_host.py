"""What the calls on drafted tokens and on 4-bit integers refuse before they touch the device, and the reference forms by hand."""
import ctypes as C
import decimal
import math
import os
import re
from fractions import Fraction

import numpy as np
import pytest
import torch

import draft_ref as ref
import paper_2511_02620_amd as difr
from paper_2511_02620_amd import binding

OK, NULL, SHAPE, DTYPE, TEMP, ALIGN, _, _, ARG = range(9)
FAKE = 0x1000                                        # never dereferenced: every call below fails validation first
MUCH = 1 << 40


def _drafts(**kw):
    r = binding._Drafts(FAKE, 0, 2, 6, 16, 16, 1.0, None, FAKE, FAKE)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _chain(**kw):
    c = binding._DraftChain(FAKE, 16, 1.0, None, FAKE, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _calls(lib):
    def chain(r, c=None, accepted=FAKE, tokens=FAKE, logp=None, flags=FAKE, ws=FAKE, n=MUCH):
        return lib.difr_draft_verify(C.byref(r), C.byref(c or _chain()), accepted, tokens, logp, flags, ws, n, None)

    def tree(r, parents=None, u=FAKE, accepted=FAKE, tokens=FAKE, nodes=FAKE, flags=FAKE, ws=FAKE, n=MUCH):
        return lib.difr_tree_verify(C.byref(r), parents, u, accepted, tokens, nodes, None, flags, ws, n, None)

    return chain, tree


def test_drafts_that_every_call_refuses():
    for call in _calls(binding.load_library()):
        for bad, want in ((dict(B=-1), SHAPE), (dict(D=-1), SHAPE), (dict(B=0), SHAPE), (dict(V=0), SHAPE), (dict(V=-1), SHAPE), (dict(ld=15), SHAPE),
                          (dict(B=1 << 31), SHAPE), (dict(D=1 << 31), SHAPE), (dict(V=1 << 31, ld=1 << 31), SHAPE), (dict(D=1 << 27), SHAPE),
                          (dict(dtype=2), DTYPE), (dict(temperature=0.0), TEMP), (dict(temperature=-1.0), TEMP),
                          (dict(temperature=float("nan")), TEMP), (dict(temperature=float("inf")), TEMP), (dict(logits=None), NULL),
                          (dict(tokens=None), NULL), (dict(offsets=None), NULL), (dict(logits=0x1001), ALIGN), (dict(dtype=1, logits=0x1002), ALIGN)):
            assert call(_drafts(**bad)) == want, (call.__name__, bad)
        for kw in (dict(accepted=None), dict(tokens=None), dict(flags=None), dict(ws=None)):
            assert call(_drafts(), **kw) == NULL, (call.__name__, kw)
        assert call(_drafts(), n=8) == SHAPE and call(_drafts(), ws=0x1010) == ALIGN
        assert call(_drafts(B=0, D=0)) == OK and call(_drafts(B=0, D=0, logits=None)) == OK


def test_arguments_of_each_call():
    lib = binding.load_library()
    chain, tree = _calls(lib)
    for kw, want in ((dict(accept_u=None), NULL), (dict(sample_u=None), NULL), (dict(ld=15), SHAPE), (dict(temperature=0.0), TEMP),
                     (dict(temperature=float("nan")), TEMP), (dict(draft=0x1001), ALIGN)):
        assert chain(_drafts(), _chain(**kw)) == want, kw
    assert lib.difr_draft_verify(C.byref(_drafts()), None, FAKE, FAKE, None, FAKE, FAKE, MUCH, None) == NULL
    assert lib.difr_draft_verify(None, C.byref(_chain()), FAKE, FAKE, None, FAKE, FAKE, MUCH, None) == NULL
    assert tree(_drafts(), u=None) == NULL and tree(_drafts(), nodes=None) == NULL


def test_workspace_sizes():
    need = binding.load_library().difr_draft_workspace_bytes
    assert need(0, 0, 10, 0, 1) == 0 and need(2, 6, 0, 0, 1) == 0 and need(2, 6, 10, 7, 1) == 0 and need(2, -1, 10, 0, 1) == 0
    assert 0 < need(2, 6, 5000, 0, 0) < need(2, 6, 5000, 0, 1) <= need(2, 7, 5000, 1, 1)
    assert need(1, 1 << 27, 16, 0, 0) == 0


def test_int4_arguments():
    lib = binding.load_library()

    def quantize(x=FAKE, dt=0, N=4, d=100, ld=100, g=64, codes=FAKE, scales=FAKE, zeros=None):
        return lib.difr_int4_quantize(x, dt, N, d, ld, g, codes, scales, zeros, None)

    def dequantize(x=FAKE, dt=0, N=4, d=100, ld=100, g=64, codes=FAKE, scales=FAKE, zeros=None):
        return lib.difr_int4_dequantize(codes, scales, zeros, N, d, g, x, dt, ld, None)

    def product(x=FAKE, dt=0, N=4, d=100, ld=100, g=64, codes=FAKE, scales=FAKE, zeros=None, V=50, out=FAKE, odt=0, ldo=50, ws=FAKE, n=1 << 40):
        return lib.difr_int4_product(x, dt, N, d, ld, codes, scales, zeros, V, g, out, odt, ldo, ws, n, None)

    for call in (quantize, dequantize, product):
        for bad, want in ((dict(N=-1), SHAPE), (dict(d=0), SHAPE), (dict(ld=99), SHAPE), (dict(N=1 << 31), SHAPE), (dict(d=1 << 24, ld=1 << 24), SHAPE),
                          (dict(g=16), ARG), (dict(g=0), ARG), (dict(g=256), ARG), (dict(dt=2), DTYPE), (dict(x=None), NULL), (dict(codes=None), NULL),
                          (dict(scales=None), NULL), (dict(x=0x1001), ALIGN), (dict(codes=0x1008), ALIGN), (dict(scales=0x1001), ALIGN)):
            assert call(**bad) == want, (call.__name__, bad)
        assert call(N=0, x=None) == OK
    for bad, want in ((dict(V=-1), SHAPE), (dict(V=1 << 31, ldo=1 << 31), SHAPE), (dict(ldo=49), SHAPE), (dict(odt=3), DTYPE), (dict(out=None), NULL),
                      (dict(out=0x1001), ALIGN), (dict(V=0), OK), (dict(N=40, n=64), SHAPE), (dict(N=40, ws=None), NULL), (dict(N=40, ws=0x1008), ALIGN)):
        assert product(**bad) == want, bad
    need = lib.difr_int4_product_workspace_bytes
    assert need(0, 64, 0, 32) == 0 and need(5, 0, 0, 32) == 0 and need(5, 64, 2, 32) == 0 and need(5, 64, 0, 33) == 0 and need(1, 4096, 0, 128) == 0
    assert 0 < need(17, 4096, 0, 128) < need(65, 4096, 0, 128) and need(17, 4096, 0, 128) < need(17, 4096, 1, 32) and need(5000, 512, 0, 64) == need(9999, 512, 0, 64)
    assert [difr.int4_padded(d) for d in (0, 1, 128, 129)] == [0, 128, 128, 256]


@pytest.mark.parametrize("bad", [None, 3, [1.0]])
def test_what_is_no_tensor_is_named(bad):
    c, s, i, f, o = (torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(3),
                     torch.tensor([0, 3]))
    for call, name in ((lambda: difr.int4_quantize(bad), "x"), (lambda: difr.int4_dequantize(bad, s, 128), "codes"),
                       (lambda: difr.int4_dequantize(c, bad, 128), "scales"), (lambda: difr.int4_product(bad, c, s), "hidden"),
                       (lambda: difr.draft_verify(bad, 1.0, i, o, f, f), "logits"), (lambda: difr.tree_verify(bad, 1.0, i, None, o, f), "logits")):
        with pytest.raises(ValueError, match="%s must be a tensor" % name):
            call()


def test_arguments_that_do_not_go_together():
    with pytest.raises(ValueError, match="group must be"):
        difr.int4_quantize(torch.zeros(2, 128), group=48)
    i, f, o, x = torch.zeros(3, dtype=torch.int32), torch.zeros(3), torch.tensor([0, 3]), torch.zeros(4, 8)
    with pytest.raises(ValueError, match="draft_temperatures"):
        difr.draft_verify(x, 1.0, i, o, f, f[:1], draft=x[:3], temperatures=torch.ones(4))
    with pytest.raises(ValueError, match="GPU tensor"):
        difr.draft_verify(x, 1.0, i, o, f, f[:1])


@pytest.mark.gpu
def test_on_the_device():
    dev = "cuda:0"
    x, i, f, o = torch.zeros(4, 8, device=dev), torch.zeros(3, dtype=torch.int32, device=dev), torch.zeros(3, device=dev), torch.tensor([0, 3], device=dev)
    q = difr.int4_quantize(x, group=32)
    for call, message in ((lambda: difr.draft_verify(x, 1.0, i, o, None, f[:1]), "accept_u must be a tensor"),
                          (lambda: difr.draft_verify(x, 1.0, i, o, f, f), "sample_u must be"),
                          (lambda: difr.draft_verify(x, 1.0, i[:2], o, f, f[:1]), "tokens must be"),
                          (lambda: difr.draft_verify(x, 1.0, i.long(), o, f, f[:1]), "tokens must be"),
                          (lambda: difr.draft_verify(x, 1.0, i, o.int(), f, f[:1]), "offsets must be"),
                          (lambda: difr.draft_verify(x, 1.0, i, o, f, f[:1], draft=x), "draft must be"),
                          (lambda: difr.draft_verify(x, 1.0, i, o, f, f[:1], draft=x[:3].bfloat16()), "draft must be"),
                          (lambda: difr.draft_verify(x, 1.0, i, o, f, f[:1], V=9), "V must be"),
                          (lambda: difr.draft_verify(x.half(), 1.0, i, o, f, f[:1]), "bfloat16 or float32"),
                          (lambda: difr.tree_verify(x, 1.0, i, i[:2], o, x[:, 0].contiguous()), "parents must be"),
                          (lambda: difr.tree_verify(x, 1.0, i, i, o, f), "sample_u must be"),
                          (lambda: difr.int4_product(x.bfloat16()[:, :0], q["codes"], q["scales"]), "hidden must be"),
                          (lambda: difr.int4_product(x, q["codes"], q["scales"].float()), "scales must be"),
                          (lambda: difr.int4_product(x, q["codes"], q["scales"], q["codes"]), "zeros must be"),
                          (lambda: difr.int4_product(x, q["codes"], q["scales"], out=x), "out must be"),
                          (lambda: difr.int4_dequantize(q["codes"], q["scales"], 129), "columns must be")):
        with pytest.raises(ValueError, match=message):
            call()
    with pytest.raises(difr.DifrError, match="temperature"):
        difr.draft_verify(x, 0.0, i, o, f, f[:1])
    with pytest.raises(difr.DifrError, match="temperature"):
        difr.tree_verify(x, -1.0, i, None, o, x[:, 0].contiguous())
    none = difr.draft_verify(x[:0], 1.0, i[:0], o[:1], f[:0], f[:0])
    assert all(t.numel() == 0 for t in none.values())


def test_the_reference_by_hand():
    p = np.array([0.5, 0.0, 0.25, 0.25])
    assert [ref.first_above(p, u) for u in (0.0, 0.49, 0.5, 0.74, 0.75, 1.0, -1.0, math.nan)] == [0, 0, 2, 2, 3, 3, 0, 0]
    assert ref.first_above(np.zeros(3), 0.5) == -1
    x = torch.tensor([[0.0, math.log(3.0)], [0.0, 0.0]])
    y = torch.tensor([[math.log(3.0), 0.0]])
    F = (1, 2, 4)
    # p = (1/4, 3/4), q = (3/4, 1/4): token 0 stands below u = 1/3, and what is left of p - q is token 1
    assert ref.draft_verify(x, [1.0, 1.0], [0], [0, 1], [0.33], [0.6], y, [1.0], F)[:2] == ([1], [0, 1])
    assert ref.draft_verify(x, [1.0, 1.0], [0], [0, 1], [0.34], [0.0], y, [1.0], F)[:2] == ([0], [1, -1])
    assert ref.draft_verify(x, [1.0, 1.0], [1], [0, 1], [0.999], [0.4], y, [1.0], F)[:2] == ([1], [1, 0])
    # without a draft's distribution token 0 stands below 1/4
    assert ref.draft_verify(x, [1.0, 1.0], [0], [0, 1], [0.24], [0.4], None, None, F)[:2] == ([1], [0, 0])
    assert ref.draft_verify(x, [1.0, 1.0], [0], [0, 1], [0.26], [0.4], None, None, F)[:2] == ([0], [1, -1])
    x = torch.zeros(4, 2)
    got = ref.tree_verify(x, [1.0] * 4, [0, 1, 1], [-1, -1, 1], [0, 3], [0.7, 0.1, 0.9, 0.2], F)
    assert got[:3] == ([2], [1, 1, 0, -1], [1, 2, -1, -1]) and got[4] == [1, 1, 0, 0]
    codes, scales, zeros, values = ref.int4(torch.tensor([[7.0, -7.0, 3.4] + [0.0] * 29]), 32, False)
    assert codes[0, 0] == 15 | 1 << 4 and scales[0, 0] == 1.0 and values[0, :3].tolist() == [7.0, -7.0, 3.0]


def test_the_polynomial_of_the_weights():
    """2^f over |f| <= 1/2, with the coefficients of the source in exact arithmetic: within 2^-45.9 of the value, so that a weight moved by two more
    such factors is good to 2^-44."""
    source = open(os.path.join(os.path.dirname(binding.__file__), "csrc", "draft_verify.hip")).read()
    body = source[source.index("double power(double d, double c)"):]
    body = body[:body.index("return")]
    first = re.search(r"double p = (0x1\.[0-9a-f]+p-\d+);", body).group(1)
    rest = re.findall(r"p = __builtin_fma\(p, f, ([^)]+)\);", body)
    coefficients = [Fraction(float.fromhex(c)) if "x" in c else Fraction(c) for c in [first] + rest]
    assert len(coefficients) == 10 and coefficients[-1] == 1
    decimal.getcontext().prec = 40
    ln2, worst = decimal.Decimal(2).ln(), decimal.Decimal(0)
    for i in range(-500, 501):
        f = Fraction(i, 1000)
        p = Fraction(0)
        for c in coefficients:
            p = p * f + c
        want = (decimal.Decimal(f.numerator) / decimal.Decimal(f.denominator) * ln2).exp()
        worst = max(worst, abs(decimal.Decimal(p.numerator) / decimal.Decimal(p.denominator) / want - 1))
    assert worst < decimal.Decimal(2) ** decimal.Decimal("-45.9"), worst
