"""4-bit matrices and distillation at sizes that choose the large tiles, and where offsets pass 32 bits."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import learn_common as LC
from paper_2402_01798_amd import binding as B
from test_gpu_mx import random_form, scratch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def on_device(values):
    return torch.from_numpy(values).cuda()


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,n,k", [(2049, 2047, 129), (2100, 2000, 1000), (3713, 3701, 300), (3900, 3800, 1), (4096, 4096, 640), (1300, 7000, 2050)])
def test_product_in_large_tiles(m, n, k, out):
    (a, va), (b, vb) = random_form(m, k, 1, 118, 122), random_form(n, k, 2, 118, 122)
    va, vb = on_device(va), on_device(vb)
    ref, size = va @ vb.t().contiguous(), va.abs() @ vb.abs().t().contiguous()
    ws = scratch(B.mx_matmul_workspace_bytes(m, n, k))
    add = torch.randn(m, n + 4, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    wide = torch.full((m, n + 3), 7.0, dtype=LC.TYPES[out], device="cuda")
    for o, extra in ((torch.empty(m, n, dtype=LC.TYPES[out], device="cuda"), None), (wide[:, :n], add[:, 1:n + 1])):
        B.tq_mx_matmul(a, b, o, ws, add=extra)
        want = ref if extra is None else ref + extra.double()
        bound = (k + 1) * 2.0 ** -23 * (size if extra is None else size + extra.double().abs()) + 1.001 * LC.HALF_ULP[out] * want.abs() \
            + (2.0 ** -25 if out == "f16" else 0.0)
        assert ((o.double() - want).abs() <= bound).all()
    assert (wide[:, n:] == 7).all()


@pytest.mark.parametrize("m,n,k", [(2100, 2000, 700), (3800, 3800, 400)])
def test_blocks_without_a_value_in_large_tiles(m, n, k):
    (a, _), (b, _) = random_form(m, k, 3), random_form(n, k, 4)
    a.scales[1, 1500, 2] = 255
    b.scales[2, 7, 0] = 255
    out = torch.empty(m, n, device="cuda")
    B.tq_mx_matmul(a, b, out, scratch(B.mx_matmul_workspace_bytes(m, n, k)))
    want = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    want[1500], want[:, 7] = True, True
    assert torch.equal(torch.isnan(out), want)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(64, 64, 8192), (70, 130, 8100), (17, 33, 20001), (300, 500, 16384), (1, 40, 200_000), (129, 65, 65_665)])
def test_product_over_a_long_axis(m, n, k, out):
    """k in parts over workgroups, joined in a second launch, whatever the workspace held."""
    (a, va), (b, vb) = random_form(m, k, 7, 118, 122), random_form(n, k, 8, 118, 122)
    nbytes = B.mx_matmul_workspace_bytes(m, n, k)
    assert nbytes > 0 and nbytes % (4 * m * n) == 0
    add = torch.randn(m, n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    for extra in (None, add):
        got = []
        for fill in (0x00, 0xFF):                           # 0xFF: NaN
            ws = torch.full((nbytes,), fill, dtype=torch.uint8, device="cuda")
            got.append(B.tq_mx_matmul(a, b, torch.full((m, n + 2), 5.0, dtype=LC.TYPES[out], device="cuda")[:, 1:n + 1], ws, extra))
        assert torch.equal(got[0], got[1])
        want = va @ vb.T + (0 if extra is None else extra.double().cpu().numpy())
        bound = LC.product_bound(va, vb, k + 1, out, want) + (0 if extra is None else (k + 1) * 2.0 ** -23 * np.abs(extra.cpu().numpy()))
        assert (np.abs(got[0].double().cpu().numpy() - want) <= bound).all()
    with pytest.raises(B.TqError) as e:
        B.tq_mx_matmul(a, b, torch.empty(m, n, device="cuda"), torch.empty(nbytes - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.code == B.EINVAL


@pytest.mark.parametrize("m,k,in_one", [(1, 177_280, True), (1, 177_281, False), (2, 32_768, True), (2, 32_769, False), (16, 2_176, True),
                                        (16, 2_177, False), (16, 11_000, False), (17, 100, False), (32, 5_000, False), (32, 6_000, False),
                                        (33, 100, False)])
def test_linear_on_both_sides_of_what_is_cast_in_the_product(m, k, in_one):
    n = 70
    w, vw = random_form(n, k, 9, 118, 122)
    nbytes = B.mx_linear_workspace_bytes(m, n, k)
    assert (nbytes == 0) == in_one
    x = torch.randn(m, k, generator=torch.Generator(device="cuda").manual_seed(m), device="cuda").bfloat16()
    out = B.tq_mx_linear(x, w, torch.empty(m, n, device="cuda"), scratch(nbytes))
    f = B.alloc_mx(m, k)
    B.tq_mx_quantize(x, f)
    vx = LC.mx_values(f.codes.cpu().numpy(), f.scales.cpu().numpy(), k)
    ref = vx @ vw.T
    assert (np.abs(out.double().cpu().numpy() - ref) <= LC.product_bound(vx, vw, k, "f32", ref)).all()


def test_cast_past_32_bits():
    """4.6e9 elements: the last rows of both forms, and of the way back."""
    rows, cols = 70_000, 65_664                             # cols: 513 groups of 128
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x[-40:] = torch.randn(40, cols, generator=g, device="cuda").bfloat16()
    x[:, -40:] = torch.randn(rows, 40, generator=g, device="cuda").bfloat16()
    f, ft = B.alloc_mx(rows, cols), B.alloc_mx(cols, rows)
    B.tq_mx_quantize(x, f, ft)
    last = x[-33:].double().cpu().numpy()
    got = f.codes[-33:, -64:].cpu().numpy()
    want, want_scales = LC.mx_form(last[:, -128:])
    assert (got == want).all() and (f.scales[-1:, -33:].cpu().numpy() == want_scales).all()
    first = rows // 128 * 128                               # the last, short group of the columns
    want, want_scales = LC.mx_form(x[first:, -33:].double().cpu().numpy().T)
    assert (ft.codes[-33:, -64:].cpu().numpy() == want).all() and (ft.scales[-1:, -33:].cpu().numpy() == want_scales).all()
    rows_only = B.alloc_mx(rows, cols)
    B.tq_mx_quantize(x, rows_only)
    assert torch.equal(rows_only.codes[-33:], f.codes[-33:]) and torch.equal(rows_only.scales[:, -33:], f.scales[:, -33:])
    del rows_only, ft
    B.tq_mx_dequantize(f, x)
    assert np.array_equal(x[-33:, -128:].double().cpu().numpy(), LC.mx_values(*LC.mx_form(last[:, -128:]), 128))


def test_product_past_32_bits():
    """An output of 4.6e9 elements, and operands with more than 2^32 codes."""
    (a, va), (b, vb) = random_form(70_000, 32, 5), random_form(66_000, 32, 6)
    out = torch.empty(70_000, 66_000, dtype=torch.bfloat16, device="cuda")
    B.tq_mx_matmul(a, b, out, scratch(B.mx_matmul_workspace_bytes(70_000, 66_000, 32)))
    for rows, cols in ((slice(0, 50), slice(0, 50)), (slice(-300, None), slice(-300, None)), (slice(65_500, 65_600), slice(-50, None))):
        ref = va[rows] @ vb[cols].T
        assert (np.abs(out[rows, cols].double().cpu().numpy() - ref) <= LC.product_bound(va[rows], vb[cols], 32, "bf16", ref)).all()
    del out
    rows, k = 9_000, 600_064                                # 5.4e9 codes, 2.7e9 bytes
    a = B.alloc_mx(rows, k)
    a.codes.zero_()
    a.scales.fill_(127)
    a.codes[-1, -1] = 0x22                                  # 1 and 1
    a.codes[-2, 0] = 0x04                                   # 2 and 0
    b = B.alloc_mx(3, k)
    b.codes.fill_(0x22)
    b.scales.fill_(128)                                     # every element 2
    out = torch.empty(rows, 3, device="cuda")
    B.tq_mx_matmul(a, b, out, scratch(B.mx_matmul_workspace_bytes(rows, 3, k)))
    assert (out[:-2] == 0).all() and (out[-1] == 4).all() and (out[-2] == 4).all()


def test_distillation_past_32_bits():
    """5.2e9 logits: the last rows."""
    rows, vocab, top = 40_000, 131_001, 16
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    z[-3:] = (3 * torch.randn(3, vocab, generator=g, device="cuda")).bfloat16()
    ids = torch.randint(0, vocab, (rows, top), generator=g, device="cuda")
    ids[-1, 0] = vocab - 1
    t = torch.randn(rows, top, generator=g, device="cuda")
    grad = torch.ones(rows, device="cuda")
    last = [v[-3:].contiguous() for v in (z, ids, t, grad)]
    want_loss, want_dz = torch.empty(3, device="cuda"), torch.empty_like(last[0])
    B.tq_distill(last[0], last[1], last[2], last[3], want_loss, want_dz)
    loss, stats = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    B.tq_distill_forward(z, ids, t, loss, stats)
    kept = z[-3:].clone()
    B.tq_distill_backward(z, ids, t, stats, grad, z)
    assert torch.allclose(loss[-3:], want_loss, rtol=1e-5) and torch.allclose(z[-3:].float(), want_dz.float(), rtol=2 ** -7, atol=1e-12)
    z[-3:] = kept
    B.tq_distill(z[-3:], ids[-3:], t[-3:], grad[-3:], loss[-3:], z[-3:])
    assert torch.allclose(z[-3:].float(), want_dz.float(), rtol=2 ** -7, atol=1e-12)
    # rows of zeros: q = 1 / vocab, less the teacher's share
    share = torch.softmax(t[5].double(), 0)
    assert abs(float(z[5].double().sum())) < 0.02 and abs(float(z[5, int(ids[5, 0])]) - (1 / vocab - float(share[ids[5] == ids[5, 0]].sum()))) < 2 ** -8


def test_with_a_folded_grid():
    """Launches beyond one grid dimension are folded; a child process lowers the fold point and runs the parity tests again."""
    from paper_2402_01798_amd import build
    assert os.path.exists(build.FOLD_TEST_LIB), "build it first: python -m paper_2402_01798_amd.build"
    env = dict(os.environ, TQ_TEST_MAX_GRID_X="40", TQ_LIBRARY_PATH=build.FOLD_TEST_LIB)
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_gpu_mx.py::test_cast",
           "tests/test_gpu_mx.py::test_product", "tests/test_gpu_mx.py::test_linear", "tests/test_gpu_learn_large.py::test_product_in_large_tiles",
           "tests/test_gpu_learn_calls.py::test_rows_in_pieces_write_what_one_workgroup_writes"]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]


@pytest.mark.parametrize("m,n,k", [(2, 40, 128), (40, 40, 128), (200, 140, 900), (64, 64, 8192), (2100, 2000, 128)])
@pytest.mark.parametrize("sa,sb", [(254, 254), (254, 127), (254, 0), (200, 200), (0, 254), (60, 60), (10, 100), (0, 0)])
def test_scales_at_the_ends_of_their_range(m, n, k, sa, sb):
    """A product that passes the range ends at infinity, one below it at its subnormal or zero; codes that meet zeros stay zero."""
    a, b = B.alloc_mx(m, k), B.alloc_mx(n, k)
    for f, scale in ((a, sa), (b, sb)):
        f.codes.zero_()
        f.scales.fill_(scale)
    a.codes[:, 0], b.codes[:, 1] = 0x07, 0x70  # 6 in columns 0 and 3: they meet zeros
    a.codes[1, 8] = b.codes[1, 8] = 0x02  # 1 in column 16 of one row of each: they meet
    out = torch.empty(m, n, device="cuda")
    B.tq_mx_matmul(a, b, out, scratch(B.mx_matmul_workspace_bytes(m, n, k)))
    want = torch.zeros(m, n)
    want[1, 1] = torch.tensor(2.0 ** (sa + sb - 254), dtype=torch.float64).float()
    assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("m,n,k", [(2051, 2045, 300), (2901, 2950, 200), (1037, 8192, 130), (1111, 8001, 130), (1500, 4001, 300), (5001, 1203, 500),
                                   (700, 1301, 300), (2047, 2040, 513), (3713, 3701, 520)])
@pytest.mark.parametrize("out,offset", [("f32", 0), ("bf16", 0), ("bf16", 3), ("f16", 1)])
def test_product_in_tiles_of_every_shape(m, n, k, out, offset):
    """Rows of the output begin at any element, and what lies between them is left alone."""
    (a, va), (b, vb) = random_form(m, k, 11, 118, 122), random_form(n, k, 12, 118, 122)
    va, vb = on_device(va), on_device(vb)
    add = torch.randn(m, n + 5, generator=torch.Generator(device="cuda").manual_seed(13), device="cuda")[:, 2:n + 2]
    ref, size = va @ vb.t().contiguous() + add.double(), va.abs() @ vb.abs().t().contiguous() + add.double().abs()
    wide = torch.full((m, n + 2 * offset + 1), 7.0, dtype=LC.TYPES[out], device="cuda")
    o = wide[:, offset:offset + n]
    B.tq_mx_matmul(a, b, o, scratch(B.mx_matmul_workspace_bytes(m, n, k)), add=add)
    bound = (k + 1) * 2.0 ** -23 * size + 1.001 * LC.HALF_ULP[out] * ref.abs() + (2.0 ** -25 if out == "f16" else 0.0)
    assert ((o.double() - ref).abs() <= bound).all()
    assert (wide[:, :offset] == 7).all() and (wide[:, offset + n:] == 7).all()


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,n,k", [(17, 33, 129), (32, 257, 1000), (3, 40, 16384), (31, 8200, 260), (5, 8300, 130), (1, 16390, 64), (33, 70, 129),
                                   (40, 100, 2000), (64, 33, 1), (63, 8190, 385), (64, 8200, 300), (20, 40, 30000)])
def test_product_of_few_rows(m, n, k, out):
    (a, va), (b, vb) = random_form(m, k, 21, 118, 122), random_form(n, k, 22, 118, 122)
    va, vb = on_device(va), on_device(vb)
    ref, size = va @ vb.t().contiguous(), va.abs() @ vb.abs().t().contiguous()
    add = torch.randn(m, n + 3, generator=torch.Generator(device="cuda").manual_seed(23), device="cuda")[:, 1:n + 1]
    ws = scratch(B.mx_matmul_workspace_bytes(m, n, k))
    for extra in (None, add):
        o = torch.full((m + 2, n + 1), 7.0, dtype=LC.TYPES[out], device="cuda")
        B.tq_mx_matmul(a, b, o[1:m + 1, :n], ws, add=extra)
        want = ref if extra is None else ref + extra.double()
        bound = (k + 1) * 2.0 ** -23 * (size if extra is None else size + extra.double().abs()) + 1.001 * LC.HALF_ULP[out] * want.abs() \
            + (2.0 ** -25 if out == "f16" else 0.0)
        assert ((o[1:m + 1, :n].double() - want).abs() <= bound).all()
        assert (o[:, n] == 7).all() and (o[0] == 7).all() and (o[m + 1] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,n,k", [(1, 50, 8192), (2, 33, 4096), (5, 130, 8192), (6, 130, 8192), (16, 64, 2048), (16, 70, 2176), (9, 8200, 384),
                                   (16, 8200, 2048), (17, 31, 1024), (16, 40, 1990), (33, 65, 640)])
def test_linear_of_few_tokens_is_the_product_of_the_cast(m, n, k, dtype):
    """Cast inside the product or before it: the same codes, so only the order of the sums is open."""
    w, vw = random_form(n, k, 31, 118, 122)
    wide = torch.randn(m, k + 5, generator=torch.Generator(device="cuda").manual_seed(32), device="cuda").to(LC.TYPES[dtype])
    for x in (wide[:, :k].contiguous(), wide[:, 3:k + 3]):
        out = torch.full((m, n + 1), 7.0, device="cuda")
        B.tq_mx_linear(x, w, out[:, :n], scratch(B.mx_linear_workspace_bytes(m, n, k)))
        form = B.alloc_mx(m, k)
        B.tq_mx_quantize(x, form)
        vx = on_device(LC.mx_values(form.codes.cpu().numpy(), form.scales.cpu().numpy(), k))
        vw_ = on_device(vw)
        ref, size = vx @ vw_.t().contiguous(), vx.abs() @ vw_.abs().t().contiguous()
        assert ((out[:, :n].double() - ref).abs() <= (k + 1) * 2.0 ** -23 * size).all()
        assert (out[:, n] == 7).all()
