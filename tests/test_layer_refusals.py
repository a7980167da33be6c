"""The calls of tq_norm.h, tq_i8.h and tq_orth.h are exported, and refuse bad arguments before touching a device."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

from paper_2402_01798_amd import binding as B
from layer_common import QUINTIC, half, i8_form, newton_schulz, pair

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
P, Q, R, S, T, ODD = (C.c_void_p(v) for v in (0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x10001))      # never dereferenced: every call below
NAN, INF = float("nan"), float("inf")                                                                      # fails its checks


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2402_01798_amd import build
        build.build()
    return B.lib()


def test_every_declared_symbol_is_exported(L):
    names = set()
    for header in ("tq_norm.h", "tq_i8.h", "tq_orth.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, header)).read(), flags=re.S)
        names |= set(re.findall(r"\b(tq_[a-z0-9_]+)\s*\(", text))
    assert names == {"tq_layernorm_forward", "tq_layernorm_backward", "tq_layernorm_workspace_bytes", "tq_i8_code_bytes", "tq_i8_quantize",
                     "tq_i8_dequantize", "tq_i8_matmul", "tq_i8_matmul_workspace_bytes", "tq_i8_linear", "tq_i8_linear_workspace_bytes",
                     "tq_orthogonalize", "tq_orthogonalize_multi", "tq_orthogonal_update", "tq_orthogonal_update_multi",
                     "tq_orthogonalize_workspace_bytes"}
    for n in names:
        assert getattr(L, n) is not None


def test_sizes(L):
    for rows, cols in ((1, 1), (3, 128), (5, 129), (1000, 1000)):
        assert L.tq_i8_code_bytes(rows, cols) == rows * -(-cols // 128) * 128
        assert L.tq_layernorm_workspace_bytes(rows, cols) >= 8 * cols
        assert L.tq_orthogonalize_workspace_bytes(rows, cols, 2, 1) == 2 * L.tq_orthogonalize_workspace_bytes(rows, cols, 1, 1) > 0
    for rows, cols in ((0, 5), (5, 0), (1 << 31, 1), (1 << 30, 1 << 20)):
        assert L.tq_i8_code_bytes(rows, cols) == 0 and L.tq_layernorm_workspace_bytes(rows, cols) == 0
        assert L.tq_orthogonalize_workspace_bytes(rows, cols, 1, 0) == 0
    assert L.tq_orthogonalize_workspace_bytes(5, 5, 0, 0) == 0 and L.tq_orthogonalize_workspace_bytes(5, 5, 65, 0) == 0
    assert L.tq_orthogonalize_workspace_bytes(5, 5, 1, 2) == 0 and L.tq_orthogonalize_workspace_bytes(32769, 32769, 1, 0) == 0
    for f in (L.tq_i8_matmul_workspace_bytes, L.tq_i8_linear_workspace_bytes):
        assert f(0, 1, 1) == 0 and f(1, 0, 1) == 0 and f(1, 1, 0) == 0 and f(1, 1, 131072) == 0


def test_layernorm_forward(L):
    def call(x=P, dtype=0, rows=4, cols=8, ldx=8, w=Q, b=Q, wtype=0, eps=1e-5, y=R, ldy=8, stats=S):
        return L.tq_layernorm_forward(x, dtype, rows, cols, ldx, w, b, wtype, eps, y, ldy, stats, None)
    for bad in (dict(x=None), dict(y=None), dict(dtype=3), dict(wtype=3), dict(rows=0), dict(cols=0), dict(ldx=7), dict(ldy=7), dict(eps=0.0),
                dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(y=P, ldy=9)):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(x=ODD), dict(y=ODD), dict(w=ODD), dict(b=ODD, wtype=1), dict(stats=C.c_void_p(0x10002))):
        assert call(**bad) == B.EALIGN, bad
    for bad in (dict(rows=1 << 31), dict(cols=1 << 31, ldx=1 << 31, ldy=1 << 31), dict(rows=1 << 20, ldx=1 << 21), dict(rows=1 << 20, ldy=1 << 21),
                dict(rows=3, ldx=(1 << 64) - 1)):
        assert call(**bad) == B.EUNSUPPORTED, bad


def test_layernorm_backward(L):
    def call(x=P, dtype=0, rows=4, cols=8, ldx=8, dy=Q, lddy=8, w=P, wtype=0, stats=S, dx=R, lddx=8, dw=S, db=S, acc=0, ws=P, nbytes=1 << 40):
        return L.tq_layernorm_backward(x, dtype, rows, cols, ldx, dy, lddy, w, wtype, stats, dx, lddx, dw, db, acc, ws, nbytes, None)
    need = L.tq_layernorm_workspace_bytes(4, 8)
    for bad in (dict(x=None), dict(dy=None), dict(stats=None), dict(dtype=3), dict(wtype=7), dict(rows=0), dict(cols=0), dict(ldx=7), dict(lddy=7), dict(lddx=7),
                dict(acc=2), dict(dx=None, dw=None, db=None), dict(dx=Q, lddx=9), dict(dx=P, lddx=9), dict(ws=None), dict(nbytes=need - 1)):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(x=ODD), dict(dy=ODD), dict(dx=ODD), dict(w=ODD), dict(stats=ODD), dict(dw=ODD), dict(db=ODD), dict(ws=ODD)):
        assert call(**bad) == B.EALIGN, bad
    for bad in (dict(rows=1 << 31), dict(rows=1 << 20, lddy=1 << 21), dict(rows=1 << 20, lddx=1 << 21)):
        assert call(**bad) == B.EUNSUPPORTED, bad


def test_i8_cast(L):
    def call(x=P, dtype=0, rows=4, cols=8, ld=8, codes=Q, scales=S):
        return L.tq_i8_quantize(x, dtype, rows, cols, ld, codes, scales, None)
    def back(codes=P, scales=S, rows=4, cols=8, out=Q, dtype=0, ldo=8):
        return L.tq_i8_dequantize(codes, scales, rows, cols, out, dtype, ldo, None)
    for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(dtype=3), dict(rows=0), dict(cols=0), dict(ld=7)):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(out=None), dict(codes=None), dict(scales=None), dict(dtype=3), dict(rows=0), dict(cols=0), dict(ldo=7)):
        assert back(**bad) == B.EINVAL, bad
    assert call(x=ODD) == call(codes=C.c_void_p(0x10008)) == call(scales=ODD) == back(out=ODD) == back(codes=ODD) == back(scales=ODD) == B.EALIGN
    for bad in (dict(rows=1 << 31), dict(rows=1 << 20, ld=1 << 21), dict(rows=1 << 30, cols=1 << 20, ld=1 << 20)):
        assert call(**bad) == B.EUNSUPPORTED, bad
    assert back(rows=1 << 31) == back(rows=1 << 20, ldo=1 << 21) == B.EUNSUPPORTED


def test_i8_matmul(L):
    def call(a=P, sa=S, b=Q, sb=S, m=4, n=8, k=16, bias=None, out=R, dtype=0, ldo=8, ws=P, nbytes=1 << 40):
        return L.tq_i8_matmul(a, sa, b, sb, m, n, k, bias, out, dtype, ldo, ws, nbytes, None)
    for name in ("a", "sa", "b", "sb", "out"):
        assert call(**{name: None}) == B.EINVAL and call(**{name: ODD}) == B.EALIGN
    for name in ("m", "n", "k"):
        assert call(**{name: 0}) == B.EINVAL and call(**{name: 1 << 31, "ldo": 1 << 31}) == B.EUNSUPPORTED
    assert call(dtype=3) == B.EINVAL and call(ldo=7) == B.EINVAL and call(bias=ODD) == B.EALIGN
    assert call(k=131072) == B.EUNSUPPORTED and call(m=1 << 20, ldo=1 << 21) == B.EUNSUPPORTED
    for m, n, k in ((64, 128, 100000), (1, 64, 131071), (300, 300, 40000)):
        need = L.tq_i8_matmul_workspace_bytes(m, n, k)
        if need:
            big = dict(m=m, n=n, k=k, ldo=n)
            assert call(**big, nbytes=need - 1) == call(**big, ws=None) == B.EINVAL and call(**big, ws=ODD) == B.EALIGN


def test_i8_linear(L):
    def call(x=P, dtype=1, m=4, ldx=16, w=Q, sw=S, n=8, k=16, bias=None, out=R, odtype=1, ldo=8, ws=P, nbytes=1 << 40):
        return L.tq_i8_linear(x, dtype, m, ldx, w, sw, n, k, bias, out, odtype, ldo, ws, nbytes, None)
    for bad in (dict(x=None), dict(w=None), dict(sw=None), dict(out=None), dict(dtype=4), dict(odtype=4), dict(m=0), dict(n=0), dict(k=0), dict(ldx=15), dict(ldo=7)):
        assert call(**bad) == B.EINVAL, bad
    assert call(x=ODD) == call(w=ODD) == call(sw=ODD) == call(out=ODD) == call(bias=ODD) == B.EALIGN
    assert call(k=131072, ldx=131072) == B.EUNSUPPORTED
    need = L.tq_i8_linear_workspace_bytes(500, 128, 1024)
    assert need > 0
    big = dict(m=500, n=128, k=1024, ldx=1024, ldo=128)
    assert call(**big, nbytes=need - 1) == call(**big, ws=None) == B.EINVAL and call(**big, ws=ODD) == B.EALIGN


def array(*ps):
    return (C.c_void_p * len(ps))(*[None if p is None else p.value for p in ps])


def test_orthogonalize(L):
    def call(g=P, dtype=0, rows=40, cols=80, steps=5, f=None, precision=1, eps=1e-7, out=Q, odtype=0, ws=R, nbytes=1 << 40):
        return L.tq_orthogonalize(g, dtype, rows, cols, steps, f, precision, eps, out, odtype, ws, nbytes, None)
    need = L.tq_orthogonalize_workspace_bytes(40, 80, 1, 1)
    for bad in (dict(g=None), dict(out=None), dict(dtype=3), dict(odtype=3), dict(rows=0), dict(cols=0), dict(steps=0), dict(steps=-1), dict(precision=2),
                dict(precision=-1), dict(eps=0.0), dict(eps=NAN), dict(eps=INF), dict(ws=None), dict(nbytes=need - 1), dict(out=P, odtype=1)):
        assert call(**bad) == B.EINVAL, bad
    assert call(g=ODD) == call(out=ODD) == call(ws=ODD) == B.EALIGN
    assert call(steps=17) == call(rows=32769, cols=32769) == call(rows=1 << 31) == call(rows=3, cols=(1 << 21) + 1) == B.EUNSUPPORTED


def test_coefficients(L):
    """Polynomials that take singular values of [0, 1] out of [-3, 3], or their factor out of 12, on any step."""
    def call(*steps):
        flat = [v for s in steps for v in s]
        # without a workspace: EINVAL for the coefficients or for that, so the coefficients are told apart by a misaligned one
        return L.tq_orthogonalize(P, 0, 40, 80, len(steps), (C.c_float * len(flat))(*flat), 1, 1e-7, Q, 0, ODD, 1 << 40, None)
    for good in ([QUINTIC] * 16, [(1.5, -0.5, 0.0)] * 16, [(1.0, 0.0, 0.0)], [(3.0, 0.0, 0.0)], [(2.0, -1.5, 0.5)] * 3, [(-1.5, 0.5, 0.0)] * 2, [(0.0, 0.0, 0.0)]):
        assert call(*good) == B.EALIGN, good
    for bad in ([(3.1, 0.0, 0.0)], [(2.0, 0.0, 0.0)] * 2, [(1.0, 2.5, 0.0)], [(0.0, 0.0, 3.5)], [(13.0, -20.0, 9.0)], [(NAN, 0.0, 0.0)], [(1.0, INF, 0.0)],
                [(1.0, 0.0, -INF)], [(8.0, -8.0, 0.0), (1.0, 0.0, 0.0)], [QUINTIC] * 3 + [(3.0, 0.0, 0.0)]):
        assert call(*bad) == B.EINVAL, bad


def test_orthogonalize_many(L):
    def call(gs, outs, count=2, dtype=0, odtype=0):
        return L.tq_orthogonalize_multi(gs, count, dtype, 40, 80, 5, None, 1, 1e-7, outs, odtype, ODD, 1 << 40, None)
    assert call(array(P, Q), array(R, S)) == B.EALIGN       # the workspace's: all else is right
    assert call(None, array(R, S)) == call(array(P, None), array(R, S)) == call(array(P, Q), array(R, S), count=0) == B.EINVAL
    assert call(array(P, Q), array(R, S), count=65) == B.EUNSUPPORTED
    def all_else(gs, outs, odtype=0):
        return L.tq_orthogonalize_multi(gs, 2, 0, 40, 80, 5, None, 1, 1e-7, outs, odtype, T, 1 << 40, None)
    assert all_else(array(P, Q), None) == all_else(array(P, Q), array(R, None)) == all_else(array(P, Q), array(R, R)) == B.EINVAL
    assert all_else(array(P, Q), array(Q, R)) == all_else(array(P, Q), array(P, R), odtype=1) == B.EINVAL


def test_update(L):
    def call(g=P, dtype=0, rows=40, cols=80, eta=0.1, mu=0.9, nesterov=1, decay=0.0, scale=1.0, steps=5, precision=1, eps=1e-7, v=Q, vo=Q, t=R, to=R, ws=T,
             nbytes=1 << 40):
        return L.tq_orthogonal_update(g, dtype, rows, cols, eta, mu, nesterov, decay, scale, steps, None, precision, eps, v, vo, t, to, ws, nbytes, None)
    need = L.tq_orthogonalize_workspace_bytes(40, 80, 1, 1)
    for bad in (dict(g=None), dict(v=None), dict(vo=None), dict(t=None), dict(to=None), dict(dtype=3), dict(rows=0), dict(nesterov=2), dict(steps=0), dict(precision=3),
                dict(eps=0.0), dict(eta=NAN), dict(eta=INF), dict(mu=NAN), dict(decay=INF), dict(scale=NAN), dict(ws=None), dict(nbytes=need - 1),
                dict(vo=R), dict(to=Q), dict(vo=P), dict(to=P), dict(vo=S, to=S), dict(vo=R, t=S, to=R)):
        assert call(**bad) == B.EINVAL, bad
    assert call(v=ODD) == call(vo=ODD) == call(t=ODD) == call(to=ODD) == call(g=ODD) == call(ws=ODD) == B.EALIGN
    many = lambda vs, vos, ts, tos, gs=array(P, C.c_void_p(0x11000)): L.tq_orthogonal_update_multi(
        gs, 2, 0, 40, 80, 0.1, 0.9, 1, 0.0, 1.0, 5, None, 1, 1e-7, vs, vos, ts, tos, T, 1 << 40, None)
    one, two = array(Q, R), array(S, C.c_void_p(0x60000))
    assert many(one, array(Q, Q), two, two) == many(one, one, two, array(S, S)) == many(one, array(R, Q), two, two) == B.EINVAL
    assert many(None, one, two, two) == many(one, None, two, two) == many(one, one, None, two) == many(one, one, two, None) == B.EINVAL


def cpu(*s, **kw):
    return torch.zeros(*s, **kw)


def test_the_binding_refuses_what_does_not_fit():
    with pytest.raises(ValueError):
        B.tq_layernorm_forward(cpu(4, 8), None, None, cpu(4, 8))               # not on a device
    with pytest.raises(TypeError):
        B.tq_layernorm_forward(cpu(4, 8, dtype=torch.float64), None, None, cpu(4, 8))
    with pytest.raises(ValueError):
        B.tq_layernorm_backward(cpu(4, 8), cpu(4, 8), None, cpu(4, 2), cpu(4, 8))
    with pytest.raises(ValueError):
        B.I8Matrix(cpu(4, 128, dtype=torch.int8), cpu(4), 4, 200)
    with pytest.raises(TypeError):
        B.I8Matrix(cpu(4, 128, dtype=torch.uint8), cpu(4), 4, 100)
    with pytest.raises(TypeError):
        B.I8Matrix(cpu(4, 128, dtype=torch.int8), cpu(4, dtype=torch.float64), 4, 100)
    with pytest.raises(ValueError):
        B.I8Matrix(cpu(4, 128, dtype=torch.int8), cpu(4), 4, 100)              # not on a device
    with pytest.raises(ValueError):
        B.tq_orthogonalize(cpu(4, 8), cpu(4, 8), None)
    with pytest.raises(ValueError):
        B.tq_orthogonalize_multi([], [], None)
    with pytest.raises(TypeError):
        B.tq_orthogonalize(cpu(4, 8, dtype=torch.int32), cpu(4, 8), None)
    with pytest.raises(ValueError):
        B._steps(2, [(1.0, 2.0, 3.0)])
    with pytest.raises(ValueError):
        B._steps(2, [(1.0, 2.0), (1.0, 2.0, 3.0, 4.0)])


def test_the_statements_that_the_kernels_are_held_to():
    """On the CPU: codes by their distances, steps that end at an orthogonal matrix, what binary16 holds of numbers."""
    codes, scales = i8_form(np.array([[1.0, 0.5, -0.25, 0.0], [0, 0, 0, 0], [127, 0.5, 1.5, -2.5]], dtype=np.float32))
    assert codes[0, :4].tolist() == [127, 64, -32, 0] and codes[2, :4].tolist() == [127, 0, 2, -2] and not codes[1].any()
    assert np.allclose(scales, [1 / 127, 0, 1])
    g = torch.randn(20, 30, dtype=torch.float64, generator=torch.Generator().manual_seed(1))
    o = newton_schulz(g, [(1.5, -0.5, 0.0)] * 40, 1e-7)
    u, _, v = torch.linalg.svd(g, full_matrices=False)
    assert torch.allclose(o, u @ v, atol=1e-9)
    x = torch.randn(1000, dtype=torch.float64)
    assert ((half(x) - x).abs() <= 2.0 ** -11 * x.abs()).all() and ((pair(x) - x).abs() <= 2.0 ** -21 * x.abs() + 2.0 ** -37).all()
