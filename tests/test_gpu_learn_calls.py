"""The example that runs the operators together; the binding's two ways into the library; capture into a graph; streams."""
import os
import sys

import pytest
import torch

import learn_common as LC
from paper_2402_01798_amd import binding as B

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_the_student_learns():
    import distill_student as D
    student, data, losses = D.train(60)
    assert losses[-1] < 0.5 * losses[0]
    student.m1.take(student.w1)
    student.m2.take(student.w2)
    # a few tokens at a time and all of them: the same casts, sums in another order, bf16 in between
    x = data[0][0]
    all_at_once = student.answer(x).float()
    for i in (0, 5, 511):
        one = student.answer(x[i:i + 1]).float()
        assert (one - all_at_once[i]).abs().max() <= 0.05 * all_at_once[i].abs().max()


def passes(seed=0):
    """One call of each function, on inputs of a few kinds; what they wrote."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(70, 300, generator=g, device="cuda").bfloat16()
    w = torch.randn(90, 300, generator=g, device="cuda")
    fx, fxt, fw = B.alloc_mx(70, 300), B.alloc_mx(300, 70), B.alloc_mx(90, 300)
    out = []
    B.tq_mx_quantize(x, fx, fxt, B.MX_STOCHASTIC, 2 ** 63 + 5, 3, 4)
    B.tq_mx_quantize(w, fw)
    B.tq_mx_quantize(x[1:2, 3:200], None, B.alloc_mx(197, 1))
    out += [fx.codes, fx.scales, fxt.codes, fxt.scales, fw.codes, fw.scales]
    out.append(B.tq_mx_dequantize(fx, torch.zeros(70, 320, device="cuda")[:, 7:307]))
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    add = torch.randn(70, 90, generator=g, device="cuda")
    out.append(B.tq_mx_matmul(fx, fw, torch.empty(70, 90, device="cuda"), ws, add))
    out.append(B.tq_mx_matmul(fx, fw, torch.empty(70, 90, device="cuda", dtype=torch.float16), ws))
    out.append(B.tq_mx_linear(x, fw, torch.empty(70, 90, device="cuda", dtype=torch.bfloat16), ws))
    out.append(B.tq_mx_linear(x[:3], fw, torch.empty(3, 90, device="cuda")))
    z = torch.randn(9, 2000, generator=g, device="cuda")
    ids = torch.randint(-1, 2000, (9, 12), generator=g, device="cuda")
    t, grad = torch.randn(9, 12, generator=g, device="cuda"), torch.rand(9, generator=g, device="cuda")
    loss, stats, dz = torch.empty(9, device="cuda"), torch.empty(9, 2, device="cuda"), torch.empty_like(z)
    B.tq_distill_forward(z, ids, t, loss, stats, 2.0)
    B.tq_distill_backward(z, ids, t, stats, grad, dz, 2.0)
    out += [loss, stats, dz]
    loss2, dz2 = torch.empty(9, device="cuda"), z.clone()
    B.tq_distill(dz2, ids.int(), t, grad, loss2, dz2, 2)
    return out + [loss2, dz2]


def equal(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


def test_the_host_module_and_the_python_code_make_the_same_calls(monkeypatch):
    taken = []
    whole = B._native_learn
    monkeypatch.setattr(B, "_native_learn", lambda name, *a: taken.append((name, whole(name, *a))) or taken[-1][1])
    first = passes()
    assert {name for name, _ in taken} == set(B._NATIVE_LEARN) and all(done for _, done in taken)
    monkeypatch.setattr(B, "_native_learn", lambda name, *a: False)
    assert equal(first, passes())


@pytest.mark.parametrize("native", [True, False])
def test_the_binding_refuses_what_does_not_fit(native, monkeypatch):
    if not native:
        monkeypatch.setattr(B, "_native_learn", lambda name, *a: False)
    dev = dict(device="cuda")
    x, f, ft = torch.zeros(8, 64, **dev), B.alloc_mx(8, 64), B.alloc_mx(64, 8)
    for call in (lambda: B.tq_mx_quantize(x, ft), lambda: B.tq_mx_quantize(x, None, f), lambda: B.tq_mx_quantize(x.t(), ft),
                 lambda: B.tq_mx_quantize(x[0], f), lambda: B.tq_mx_quantize(x.cpu(), f), lambda: B.tq_mx_dequantize(f, x.t()),
                 lambda: B.tq_mx_dequantize(f, torch.zeros(8, 63, **dev)), lambda: B.tq_mx_matmul(f, ft, torch.zeros(8, 64, **dev)),
                 lambda: B.tq_mx_matmul(f, f, torch.zeros(8, 9, **dev)), lambda: B.tq_mx_linear(x, ft, torch.zeros(8, 64, **dev)),
                 lambda: B.tq_mx_matmul(f, f, torch.zeros(8, 8, **dev), None, torch.zeros(8, 9, **dev)),
                 lambda: B.MxMatrix(f.codes[:, :32], f.scales, 8, 64), lambda: B.MxMatrix(f.codes.cpu(), f.scales, 8, 64)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.tq_mx_quantize(x.double(), f), lambda: B.tq_mx_dequantize(f, x.int())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: B.tq_mx_quantize(x, None, None), lambda: B.tq_mx_quantize(x, f, None, 7),
                 lambda: B.tq_mx_dequantize(f, torch.zeros(8, 64, dtype=torch.float16, **dev)),
                 lambda: B.tq_mx_quantize(torch.zeros(0, 64, **dev), None, None)):
        with pytest.raises(B.TqError) as e:
            call()
        assert e.value.code == B.EINVAL
    z, ids, t, row = torch.zeros(4, 50, **dev), torch.zeros(4, 3, dtype=torch.int32, **dev), torch.zeros(4, 3, **dev), torch.zeros(4, **dev)
    stats = torch.zeros(4, 2, **dev)
    for call in (lambda: B.tq_distill_forward(z, ids[:3], t, row, stats), lambda: B.tq_distill_forward(z, ids, t[:, :2], row, stats),
                 lambda: B.tq_distill_forward(z, ids, t, row, row), lambda: B.tq_distill_backward(z, ids, t, stats, row[:3], z),
                 lambda: B.tq_distill(z, ids, t, row, row, torch.zeros(4, 49, **dev)), lambda: B.tq_distill(z, ids, t, row, row, z.half())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.tq_distill_forward(z, ids.short(), t, row, stats), lambda: B.tq_distill_forward(z, ids, t.half(), row, stats),
                 lambda: B.tq_distill(z, ids, t, row.double(), row, z)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(B.TqError):
        B.tq_distill_forward(z, ids, t, row, stats, 0.0)
    with pytest.raises(B.TqError):
        B.tq_distill_forward(z, torch.zeros(4, 1025, dtype=torch.int32, **dev), torch.zeros(4, 1025, **dev), row, stats)


def test_calls_replay_from_a_graph():
    """Captured once, replayed several times with other work between the replays: each replay gives the eager results."""
    want = [t.clone() for t in passes(1)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x = torch.randn(70, 300, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
        w = torch.randn(90, 300, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
        fx, fxt, fw, ws = B.alloc_mx(70, 300), B.alloc_mx(300, 70), B.alloc_mx(90, 300), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        y, y1, z = torch.empty(70, 90, device="cuda"), torch.empty(1, 90, device="cuda"), torch.empty(70, 90, device="cuda")
        ids = torch.arange(5, device="cuda").repeat(70, 1)
        t, grad, loss, dz = torch.randn(70, 5, device="cuda"), torch.ones(70, device="cuda"), torch.empty(70, device="cuda"), torch.empty_like(y)

        def work():
            B.tq_mx_quantize(x, fx, fxt, B.MX_STOCHASTIC, 1, 2, 3)
            B.tq_mx_quantize(w, fw)
            B.tq_mx_matmul(fx, fw, y, ws)
            B.tq_mx_linear(x[:1], fw, y1)
            B.tq_distill(y, ids, t, grad, loss, dz)

        work()
        torch.cuda.synchronize()
        eager = [v.clone() for v in (fx.codes, fxt.codes, y, y1, loss, dz)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            work()
        for _ in range(4):
            for v in (fx.codes, fxt.codes, y, y1, loss, dz):
                v.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert equal(eager, (fx.codes, fxt.codes, y, y1, loss, dz))
            assert equal(want, passes(1))


@pytest.mark.parametrize("rows,vocab", [(1, 40000), (5, 131001), (40, 70000)])
def test_rows_in_pieces_write_what_one_workgroup_writes(rows, vocab):
    """Few rows are split over workgroups in the backward pass, many are not: the same bits for the same row."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    z = torch.randn(rows, vocab, generator=g, device="cuda").bfloat16()
    ids = torch.randint(0, vocab, (rows, 30), generator=g, device="cuda")
    ids[:, 7] = ids[:, 3]
    t, grad = torch.randn(rows, 30, generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda")
    many = -(-1100 // rows)
    big = [v.repeat(many, 1).contiguous() if v.dim() == 2 else v.repeat(many) for v in (z, ids, t, grad)]
    got = []
    for a, b, c, d in ((z, ids, t, grad), big):
        loss, stats, dz = torch.empty(a.shape[0], device="cuda"), torch.empty(a.shape[0], 2, device="cuda"), a.clone()
        B.tq_distill_forward(a, b, c, loss, stats)
        B.tq_distill_backward(dz, b, c, stats, d, dz)
        got.append(dz)
    aligned = [i for i in range(rows) if (i * vocab) % 8 == 0]                # (a row's place decides which elements are loose)
    for copy in (0, many - 1):
        part = got[1][copy * rows:(copy + 1) * rows]
        assert torch.equal(part[aligned], got[0][aligned]) if copy == 0 else torch.allclose(part.float(), got[0].float(), rtol=2 ** -7)
