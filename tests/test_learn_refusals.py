"""The calls of tq_mx.h and tq_distill.h are exported, and refuse bad arguments before touching a device."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2402_01798_amd import binding as B

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
P, ODD = C.c_void_p(0x10000), C.c_void_p(0x10001)          # never dereferenced: every call below fails its checks


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2402_01798_amd import build
        build.build()
    return B.lib()


def test_every_declared_symbol_is_exported(L):
    names = set()
    for header in ("tq_mx.h", "tq_distill.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, header)).read(), flags=re.S)
        names |= set(re.findall(r"\b(tq_[a-z_]+)\s*\(", text))
    assert names == {"tq_mx_code_bytes", "tq_mx_scale_bytes", "tq_mx_quantize", "tq_mx_dequantize", "tq_mx_matmul",
                     "tq_mx_matmul_workspace_bytes", "tq_mx_linear", "tq_mx_linear_workspace_bytes", "tq_distill",
                     "tq_distill_forward", "tq_distill_backward"}
    for n in names:
        assert getattr(L, n) is not None


def test_sizes(L):
    for rows, cols in ((1, 1), (3, 128), (5, 129), (1000, 1000)):
        groups = -(-cols // 128)
        assert L.tq_mx_code_bytes(rows, cols) == rows * groups * 64
        assert L.tq_mx_scale_bytes(rows, cols) == rows * groups * 4
    for rows, cols in ((0, 5), (5, 0), (1 << 31, 1), (1 << 30, 1 << 20)):
        assert L.tq_mx_code_bytes(rows, cols) == 0 and L.tq_mx_scale_bytes(rows, cols) == 0
    assert L.tq_mx_matmul_workspace_bytes(0, 1, 1) == 0 and L.tq_mx_linear_workspace_bytes(1, 1, 0) == 0


def test_quantize(L):
    def call(x=P, dtype=0, rows=4, cols=8, ld=8, rounding=0, forms=(P, P, P, P)):
        return L.tq_mx_quantize(x, dtype, rows, cols, ld, rounding, 0, 0, 0, *forms, None)
    assert call(x=None) == B.EINVAL
    assert call(dtype=3) == B.EINVAL
    assert call(rows=0) == B.EINVAL and call(cols=0, ld=0) == B.EINVAL
    assert call(ld=7) == B.EINVAL
    assert call(rounding=2) == B.EINVAL
    assert call(forms=(None, None, None, None)) == B.EINVAL
    assert call(forms=(P, None, P, P)) == B.EINVAL and call(forms=(P, P, None, P)) == B.EINVAL
    assert call(x=ODD, dtype=1) == B.EALIGN
    assert call(forms=(P, ODD, None, None)) == B.EALIGN and call(forms=(None, None, ODD, P)) == B.EALIGN
    assert call(rows=1 << 31) == B.EUNSUPPORTED
    assert call(rows=1 << 20, ld=1 << 21) == B.EUNSUPPORTED
    assert call(rows=3, ld=(1 << 64) - 1) == B.EUNSUPPORTED


def test_dequantize(L):
    def call(codes=P, scales=P, rows=4, cols=8, out=P, dtype=0, ldo=8):
        return L.tq_mx_dequantize(codes, scales, rows, cols, out, dtype, ldo, None)
    assert call(codes=None) == B.EINVAL and call(out=None) == B.EINVAL
    assert call(dtype=2) == B.EINVAL                       # fp16 does not hold the range
    assert call(ldo=7) == B.EINVAL and call(rows=0) == B.EINVAL
    assert call(scales=ODD) == B.EALIGN and call(out=ODD) == B.EALIGN
    assert call(rows=1 << 31) == B.EUNSUPPORTED


def test_matmul(L):
    def call(a=P, sa=P, b=P, sb=P, m=4, n=8, k=16, add=None, lda=8, out=P, dtype=0, ldo=8, ws=P, nbytes=1 << 40):
        return L.tq_mx_matmul(a, sa, b, sb, m, n, k, add, lda, out, dtype, ldo, ws, nbytes, None)
    for name in ("a", "sa", "b", "sb"):
        assert call(**{name: None}) == B.EINVAL
        assert call(**{name: ODD}) == B.EALIGN
    assert call(out=None) == B.EINVAL and call(out=ODD) == B.EALIGN and call(dtype=5) == B.EINVAL
    for name in ("m", "n", "k"):
        assert call(**{name: 0}) == B.EINVAL
        assert call(**{name: 1 << 31, "ldo": 1 << 31}) == B.EUNSUPPORTED
    assert call(ldo=7) == B.EINVAL
    assert call(add=C.c_void_p(0x20000), lda=7) == B.EINVAL and call(add=ODD) == B.EALIGN
    assert call(add=P, dtype=1) == B.EINVAL                # added in place: floats
    assert call(add=P, lda=9) == B.EINVAL                  # and the same rows
    need = L.tq_mx_matmul_workspace_bytes(64, 128, 1 << 16)
    if need:
        big = dict(m=64, n=128, k=1 << 16, ldo=128)
        assert call(**big, nbytes=need - 1) == B.EINVAL and call(**big, ws=None) == B.EINVAL and call(**big, ws=ODD) == B.EALIGN


def test_linear(L):
    def call(x=P, dtype=1, m=4, ldx=16, w=P, sw=P, n=8, k=16, out=P, odtype=1, ldo=8, ws=P, nbytes=1 << 40):
        return L.tq_mx_linear(x, dtype, m, ldx, w, sw, n, k, out, odtype, ldo, ws, nbytes, None)
    assert call(x=None) == B.EINVAL and call(w=None) == B.EINVAL and call(out=None) == B.EINVAL
    assert call(dtype=4) == B.EINVAL and call(odtype=4) == B.EINVAL
    assert call(m=0) == B.EINVAL and call(n=0) == B.EINVAL and call(k=0) == B.EINVAL
    assert call(ldx=15) == B.EINVAL and call(ldo=7) == B.EINVAL
    assert call(x=ODD) == B.EALIGN and call(sw=ODD) == B.EALIGN
    need = L.tq_mx_linear_workspace_bytes(500, 128, 1024)
    assert need > 0
    big = dict(m=500, n=128, k=1024, ldx=1024, ldo=128)
    assert call(**big, nbytes=need - 1) == B.EINVAL and call(**big, ws=None) == B.EINVAL and call(**big, ws=ODD) == B.EALIGN


def test_distill(L):
    def args(z=P, dtype=0, rows=4, vocab=100, ldz=100, ids=P, id_bytes=4, t=P, top=5, tau=1.0):
        return z, dtype, rows, vocab, ldz, ids, id_bytes, t, top, tau
    bad = [dict(z=None), dict(dtype=3), dict(rows=0), dict(vocab=0), dict(ldz=99), dict(ids=None), dict(id_bytes=2), dict(t=None),
           dict(top=0), dict(tau=0.0), dict(tau=float("nan")), dict(tau=-1.0), dict(tau=float("inf"))]
    other = C.c_void_p(0x20000)
    for code, changes in [(B.EINVAL, c) for c in bad] + [(B.EALIGN, dict(z=ODD)), (B.EALIGN, dict(ids=C.c_void_p(0x10004), id_bytes=8)),
                                                         (B.EALIGN, dict(t=ODD)), (B.EUNSUPPORTED, dict(top=1025)),
                                                         (B.EUNSUPPORTED, dict(rows=1 << 31))]:
        a = args(**changes)
        assert L.tq_distill_forward(*a, P, P, None) == code, changes
        assert L.tq_distill_backward(*a, P, P, other, 1 << 10, None) == code, changes
        assert L.tq_distill(*a, P, P, other, 1 << 10, None) == code, changes
    a = args()
    assert L.tq_distill_forward(*a, None, P, None) == B.EINVAL and L.tq_distill_forward(*a, P, ODD, None) == B.EALIGN
    for f in (L.tq_distill_backward, L.tq_distill):
        assert f(*a, None, P, other, 100, None) == B.EINVAL and f(*a, P, None, other, 100, None) == B.EINVAL
        assert f(*a, P, P, None, 100, None) == B.EINVAL and f(*a, P, P, other, 99, None) == B.EINVAL
        assert f(*a, P, P, P, 101, None) == B.EINVAL       # in place: the same rows
        assert f(*a, P, P, ODD, 100, None) == B.EALIGN


def test_the_binding_refuses_what_does_not_fit():
    cpu = lambda *s, **kw: torch.zeros(*s, **kw)
    with pytest.raises(ValueError):
        B.tq_mx_quantize(cpu(4, 8), None, None)             # not on a device
    with pytest.raises(TypeError):
        B.tq_mx_quantize(cpu(4, 8, dtype=torch.float64), None, None)
    with pytest.raises(ValueError):
        B.tq_mx_quantize(cpu(8), None, None)
    with pytest.raises(ValueError):
        B.MxMatrix(cpu(4, 64, dtype=torch.uint8), cpu(1, 4, 4, dtype=torch.uint8), 4, 200)
    with pytest.raises(TypeError):
        B.MxMatrix(cpu(4, 64), cpu(1, 4, 4, dtype=torch.uint8), 4, 100)
    with pytest.raises(ValueError):
        B.tq_distill_forward(cpu(4, 8), cpu(4, 2, dtype=torch.int32), cpu(4, 2), cpu(4), cpu(4))
