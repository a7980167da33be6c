"""Layer norm, 8-bit matrices and orthogonalised updates together and with the calls that stand beside them; the binding's two ways into the
library; streams, graphs, sizes past 32 bits, folded grids."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2402_01798_amd import binding as B
from layer_common import HALF_ULP, QUINTIC, U, i8_form, i8_product, newton_schulz, newton_schulz_bound, norm_backward, norm_backward_bounds, norm_forward, norm_forward_bound

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def workspace(nbytes):
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")


def inputs(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return {"x": n(70, 300).bfloat16(), "dy": n(70, 300).bfloat16(), "w": 1 + 0.1 * n(300), "b": n(300), "weights": n(90, 300), "bias": n(90),
            "g": n(96, 130) * 1e-3, "v": n(96, 130) * 1e-2, "t": n(96, 130), "g2": n(200, 150)}


def buffers():
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")
    return {"y": e(70, 300, dtype=torch.bfloat16), "stats": e(70, 2), "dx": e(70, 300, dtype=torch.bfloat16), "dw": e(300), "db": e(300), "fx": B.alloc_i8(70, 300),
            "fw": B.alloc_i8(90, 300), "values": e(70, 320)[:, 7:307], "out": e(70, 90), "out2": e(70, 90, dtype=torch.float16), "out3": e(3, 90, dtype=torch.bfloat16),
            "v2": e(96, 130), "t2": e(96, 130), "o": e(200, 150, dtype=torch.bfloat16), "ws": workspace(1 << 24)}


def passes(i, b):
    """One call of each function; what they wrote."""
    B.tq_layernorm_forward(i["x"], i["w"], i["b"], b["y"], b["stats"], 1e-6)
    B.tq_layernorm_backward(i["x"], i["dy"], i["w"], b["stats"], b["dx"], b["dw"], b["db"], b["ws"])
    B.tq_i8_quantize(b["y"], b["fx"])
    B.tq_i8_quantize(i["weights"], b["fw"])
    B.tq_i8_dequantize(b["fx"], b["values"])
    B.tq_i8_matmul(b["fx"], b["fw"], b["out"], b["ws"], i["bias"])
    B.tq_i8_linear(b["y"], b["fw"], b["out2"], b["ws"])
    B.tq_i8_linear(b["y"][:3], b["fw"], b["out3"], b["ws"], bias=i["bias"])
    B.tq_orthogonal_update(i["g"], i["v"], i["t"], b["ws"], eta=0.1, velocity_out=b["v2"], theta_out=b["t2"])
    B.tq_orthogonalize(i["g2"], b["o"], b["ws"])
    return [b[k] for k in ("y", "stats", "dx", "dw", "db", "values", "out", "out2", "out3", "v2", "t2", "o")] + [b["fx"].codes, b["fx"].scales, b["fw"].codes]


def copies(ts):
    return [t.clone() for t in ts]


def equal(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


def test_the_host_module_and_the_python_code_make_the_same_calls(monkeypatch):
    taken = []
    whole = B._native_layer
    monkeypatch.setattr(B, "_native_layer", lambda name, *a: taken.append((name, whole(name, *a))) or taken[-1][1])
    first = copies(passes(inputs(), buffers()))
    assert {name for name, _ in taken} == set(B._NATIVE_LAYER) and all(done for _, done in taken)
    monkeypatch.setattr(B, "_native_layer", lambda name, *a: False)
    assert equal(passes(inputs(), buffers()), first)


@pytest.mark.parametrize("native", [True, False])
def test_what_does_not_fit_is_refused(monkeypatch, native):
    if not native:
        monkeypatch.setattr(B, "_native_layer", lambda name, *a: False)
    i, b = inputs(), buffers()
    x, y, w, ws = i["x"], b["y"], i["w"], b["ws"]
    for bad, kind in (((x, w, None, y.float()), ValueError), ((x, w, None, y[:69]), ValueError), ((x, w[:299], None, y), ValueError), ((x, w, w.bfloat16(), y), TypeError),
                      ((x, w.cpu(), None, y), ValueError), ((x, w, None, y.cpu()), ValueError), ((x.t(), None, None, y.t()), ValueError),
                      ((x, w, None, y, b["stats"][:69]), ValueError), ((x, w, None, y, b["stats"].double()), TypeError), ((x.double(), w, None, y), TypeError)):
        with pytest.raises(kind):
            B.tq_layernorm_forward(*bad)
    for bad in ((x, i["dy"], w, None, b["dx"]), (x, i["dy"], w, b["stats"], b["dx"], b["dw"], b["db"]), (x, i["dy"], w, b["stats"], None),
                (x, i["dy"], w, b["stats"], b["dx"], b["dw"], None, ws[:64])):
        with pytest.raises(B.TqError):
            B.tq_layernorm_backward(*bad)
    for bad in ((x, i["dy"][:, :299], w, b["stats"], b["dx"]), (x, i["dy"], w, b["stats"], b["dx"], b["dw"][:5], None, ws)):
        with pytest.raises(ValueError):
            B.tq_layernorm_backward(*bad)
    with pytest.raises(ValueError):
        B.tq_i8_quantize(x, b["fw"])
    with pytest.raises(ValueError):
        B.tq_i8_matmul(b["fx"], b["fw"], b["out"].t(), ws)
    with pytest.raises(ValueError):
        B.tq_i8_matmul(b["fx"], b["fw"], b["out"], ws, i["bias"][:5])
    with pytest.raises(TypeError):
        B.tq_i8_linear(y, b["fw"], b["out"], ws, bias=i["bias"].double())
    with pytest.raises(B.TqError):
        B.tq_i8_linear(y, b["fw"], b["out"], None)
    for bad, kind in (((i["g"], i["g"][:, :5], ws), ValueError), ((i["g"].t(), b["v2"], ws), ValueError), ((i["g"], b["v2"], ws[:100]), B.TqError), ((i["g"], b["v2"], None), B.TqError)):
        with pytest.raises(kind):
            B.tq_orthogonalize(*bad)
    with pytest.raises(TypeError):
        B.tq_orthogonal_update(i["g"], i["v"].bfloat16(), i["t"], ws, eta=0.1)
    with pytest.raises(B.TqError):
        B.tq_orthogonal_update(i["g"], i["v"], i["v"], ws, eta=0.1)             # momentum and parameters in one buffer


def test_another_stream():
    want = copies(passes(inputs(3), buffers()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    i, b = inputs(3), buffers()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = passes(i, b)
    side.synchronize()
    assert equal(got, want)


def test_captured_and_replayed_with_other_inputs():
    i, b = inputs(1), buffers()
    passes(i, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = passes(i, b)
    for seed in (5, 6, 7):
        fresh = inputs(seed)
        want = copies(passes(fresh, buffers()))
        for k in i:
            i[k].copy_(fresh[k])
        for t in got:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert equal(got, want)


def test_a_training_step_and_an_answer():
    """Worker: norm, 4-bit layer, distillation, gradients back through both; the gradients compressed and averaged; the server's update of
    the matrix; the student's answer in 8 bits.  Every link against 64 bits on what it was given."""
    g = torch.Generator(device="cuda").manual_seed(11)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    tokens, width, vocab, top, bits = 96, 256, 384, 8, 4
    theta = torch.empty(vocab * width + 2 * width, device="cuda")                # the layer's weights, the norm's weight and bias
    w, gamma, beta = theta[:vocab * width].view(vocab, width), theta[vocab * width:-width], theta[-width:]
    w.copy_(n(vocab, width) * width ** -0.5)
    gamma.copy_(1 + 0.1 * n(width))
    beta.copy_(0.1 * n(width))
    gradients, ws = [torch.empty_like(theta) for _ in range(2)], workspace(1 << 25)
    for worker, gradient in enumerate(gradients):
        x = n(tokens, width).bfloat16()
        t, ids = torch.topk(n(tokens, vocab), top, dim=1)
        y, stats = torch.empty_like(x), torch.empty(tokens, 2, device="cuda")
        B.tq_layernorm_forward(x, gamma, beta, y, stats)
        fy, fyt, fw, fwt, fz, fzt = (B.alloc_mx(*s) for s in ((tokens, width), (width, tokens), (vocab, width), (width, vocab), (tokens, vocab), (vocab, tokens)))
        B.tq_mx_quantize(y, fy, fyt)
        B.tq_mx_quantize(w, fw, fwt)
        z = B.tq_mx_matmul(fy, fw, torch.empty(tokens, vocab, dtype=torch.bfloat16, device="cuda"), ws)
        loss = torch.empty(tokens, device="cuda")
        B.tq_distill(z, ids, t, torch.full((tokens,), 1 / tokens, device="cuda"), loss, z, 2.0)
        B.tq_mx_quantize(z, fz, fzt, B.MX_STOCHASTIC, 100 + worker, worker, 0)
        B.tq_mx_matmul(fzt, fyt, gradient[:vocab * width].view(vocab, width), ws)
        dy = B.tq_mx_matmul(fz, fwt, torch.empty_like(y), ws)
        dx = torch.empty_like(x)
        B.tq_layernorm_backward(x, dy, gamma, stats, dx, gradient[vocab * width:-width], gradient[-width:], ws)
        x64, dy64, w64 = x.double(), dy.double(), gamma.double()
        want, h, mean, r = norm_forward(x64, w64, beta.double(), 1e-5)
        assert ((y.double() - want).abs() <= norm_forward_bound(want, h, w64, beta.double(), width, "bf16")).all()
        for got, t64, far in zip((dx, gradient[vocab * width:-width], gradient[-width:]), norm_backward(dy64, h, w64, r),
                                 norm_backward_bounds(x64, dy64, h, w64, mean, r, "bf16", tokens + 40)):
            assert ((got.double() - t64).abs() <= far).all()
        assert loss.isfinite().all()
    d = theta.numel()
    stats, params, payloads = [B.alloc_stats(d) for _ in gradients], [B.alloc_params(d) for _ in gradients], [B.alloc_payload(d, bits) for _ in gradients]
    B.tq_stats_multi(gradients, stats, workspace(2 * B.stats_workspace_bytes(d)))
    B.tq_params_multi(stats, params, bits, B.GRID_UNIFORM)
    B.tq_compress_multi(gradients, params, payloads, bits, 1, 0, 0, grid=B.GRID_UNIFORM)
    average = torch.empty(d, device="cuda")
    B.tq_decompress_aggregate(payloads, params, average, bits)
    ghost, before, velocity = average[:vocab * width].view(vocab, width), w.clone(), torch.zeros(vocab, width, device="cuda")
    B.tq_orthogonal_update(ghost, velocity, w, ws, eta=0.02, weight_decay=0.1, scale=(vocab / width) ** 0.5)
    mu = float(torch.tensor(0.95))
    u = ghost.double() + mu * ghost.double()
    o = newton_schulz(u, [QUINTIC] * 5, 1e-7)
    want = before.double() - float(torch.tensor(0.02)) * (float(torch.tensor((vocab / width) ** 0.5)) * o + float(torch.tensor(0.1)) * before.double())
    off = 0.02 * 1.3 * newton_schulz_bound(u, [QUINTIC] * 5, 1e-7, 2.0 ** -21 + 8 * U, (vocab + 8) * U) + 6 * U * float(want.norm() + before.norm())
    assert float((w.double() - want).norm()) <= off and torch.equal(velocity, ghost)
    f8 = B.tq_i8_quantize(w, B.alloc_i8(vocab, width))
    answer = B.tq_i8_linear(y[:5], f8, torch.empty(5, vocab, device="cuda"), ws)
    codes, scales = i8_form(y[:5].float().cpu().numpy())
    assert torch.equal(answer.cpu(), i8_product(codes, scales, f8.codes.cpu().numpy(), f8.scales.cpu().numpy(), None, "f32"))


# ---- sizes past 32 bits

def far_rows(rows, cols, ld, dtype):
    """`rows` rows that are `ld` elements apart."""
    return torch.empty((rows - 1) * ld + cols, dtype=dtype, device="cuda").as_strided((rows, cols), (ld, 1))


def test_rows_past_32_bits():
    rows, cols, ld = 3, 1000, (1 << 31) + 24
    g = torch.Generator(device="cuda").manual_seed(2)
    near = torch.randn(rows, cols, generator=g, device="cuda").bfloat16()
    x, y = far_rows(rows, cols, ld, torch.bfloat16), far_rows(rows, cols, ld, torch.bfloat16)
    x.copy_(near)
    stats, stats2, near_y, near_dx = torch.empty(rows, 2, device="cuda"), torch.empty(rows, 2, device="cuda"), torch.empty_like(near), torch.empty_like(near)
    B.tq_layernorm_forward(x, None, None, y, stats)
    B.tq_layernorm_forward(near, None, None, near_y, stats2)
    assert torch.equal(y, near_y) and torch.equal(stats, stats2)
    B.tq_layernorm_backward(x, x, None, stats, y)
    B.tq_layernorm_backward(near, near, None, stats, near_dx)
    assert torch.equal(y, near_dx)
    f, f2 = B.tq_i8_quantize(x, B.alloc_i8(rows, cols)), B.tq_i8_quantize(near, B.alloc_i8(rows, cols))
    assert torch.equal(f.codes, f2.codes) and torch.equal(f.scales, f2.scales)
    B.tq_i8_dequantize(f, y)
    assert torch.equal(y, (f.codes[:, :cols].float() * f.scales.view(-1, 1)).bfloat16())
    w = B.tq_i8_quantize(torch.randn(200, cols, generator=g, device="cuda"), B.alloc_i8(200, cols))
    out, near_out = far_rows(rows, 200, ld, torch.bfloat16), torch.empty(rows, 200, dtype=torch.bfloat16, device="cuda")
    B.tq_i8_linear(x, w, out, workspace(B.i8_linear_workspace_bytes(rows, 200, cols)))
    B.tq_i8_linear(near, w, near_out, workspace(B.i8_linear_workspace_bytes(rows, 200, cols)))
    assert torch.equal(out, near_out)
    many, near_many = far_rows(40, 200, 1 << 27, torch.float32), torch.empty(40, 200, device="cuda")
    a = B.tq_i8_quantize(torch.randn(40, cols, generator=g, device="cuda"), B.alloc_i8(40, cols))
    ws = workspace(B.i8_matmul_workspace_bytes(40, 200, cols))
    assert torch.equal(B.tq_i8_matmul(a, w, many, ws), B.tq_i8_matmul(a, w, near_many, ws))


@pytest.mark.parametrize("m", [1, 20, 50])
def test_codes_past_32_bits(m):
    n, k = 1_100_000, 4096
    g = torch.Generator(device="cuda").manual_seed(m)
    w = torch.empty(n, k, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    fw = B.tq_i8_quantize(w, B.alloc_i8(n, k))
    tail = slice(n - 500, n)
    part = B.tq_i8_quantize(w[tail], B.alloc_i8(500, k))
    assert torch.equal(fw.codes[tail], part.codes) and torch.equal(fw.scales[tail], part.scales)
    B.tq_i8_dequantize(fw, w)
    assert torch.equal(w[tail], (part.codes.float() * part.scales.view(-1, 1)).bfloat16())
    x = torch.randn(m, k, generator=g, device="cuda")
    out, want = torch.empty(m, n, device="cuda"), torch.empty(m, 500, device="cuda")
    B.tq_i8_linear(x, fw, out, workspace(B.i8_linear_workspace_bytes(m, n, k)))
    B.tq_i8_linear(x, part, want, workspace(B.i8_linear_workspace_bytes(m, 500, k)))
    assert torch.equal(out[:, tail], want)


def test_many_elements_in_a_norm():
    rows, cols = 70_000, 65_536
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    y, stats, dx = torch.empty_like(x), torch.empty(rows, 2, device="cuda"), torch.empty_like(x)
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    B.tq_layernorm_forward(x, None, None, y, stats)
    B.tq_layernorm_backward(x, x, None, stats, dx, dw, db, workspace(B.layernorm_workspace_bytes(rows, cols)))
    for part in (slice(0, 3), slice(rows - 3, rows)):
        few, few_stats = torch.empty(3, cols, dtype=torch.bfloat16, device="cuda"), torch.empty(3, 2, device="cuda")
        B.tq_layernorm_forward(x[part], None, None, few, few_stats)
        assert torch.equal(y[part], few) and torch.equal(stats[part], few_stats)
        B.tq_layernorm_backward(x[part], x[part], None, few_stats, few)
        assert torch.equal(dx[part], few)
    want = sum(c.double().sum(dim=0) for c in x.split(10_000))
    assert ((db.double() - want).abs() <= (rows // 64 + 44) * U * 1.01 * rows).all()      # normal numbers: a mean magnitude below 1.01


@pytest.mark.parametrize("rows, precision", [(1040, B.ORTH_HALF), (520, B.ORTH_SPLIT)])
def test_a_long_matrix_past_32_bits(rows, precision):
    """X has 2^32 bytes and more, 256 of its rows 2^31.  With F_i the factors of the steps, all polynomials of G G^T / |G|^2, the result is
    F_5 ... F_1 G / |G|."""
    cols = B.ORTH_MAX_LENGTH
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out = torch.empty_like(x)
    B.tq_orthogonalize(x, out, workspace(B.orthogonalize_workspace_bytes(rows, cols, 1, precision)), precision=precision)
    gram = sum((c @ c.t().contiguous() for c in (p.double() for p in x.split(1 << 17, dim=1))), torch.zeros(rows, rows, dtype=torch.float64, device="cuda"))
    size = gram.diagonal().sum().sqrt() + 1e-7
    gram, all_factors, one = gram / size ** 2, torch.eye(rows, dtype=torch.float64, device="cuda"), torch.eye(rows, dtype=torch.float64, device="cuda")
    for _ in range(5):
        a, b, c = QUINTIC
        factor = a * one + b * gram + c * (gram @ gram)
        all_factors, gram = factor @ all_factors, factor @ gram @ factor
    # all singular values are alike (within 5 %): errors are not lifted beyond the values, 15 roundings of 2^-11 with slopes up to 4 between
    # steps would be 2^-11 * 15 * 4 at most for the two steps that still turn, and bf16's own half step
    held = 2.0 ** -11 if precision == B.ORTH_HALF else 2.0 ** -16      # pairs: sums of 2^21 terms, sqrt(2^21) 2^-24 each beside 2^-21
    for part in (slice(0, 300), slice(cols - 300, cols)):
        want = all_factors @ (x[:, part].double() / size)
        far = (out[:, part].double() - want).norm(dim=1)
        assert (far <= (60 * held + HALF_ULP["bf16"]) * want.norm(dim=1)).all()


def test_with_a_folded_grid():
    from paper_2402_01798_amd import build
    assert os.path.exists(build.FOLD_TEST_LIB), "build it first: python -m paper_2402_01798_amd.build"
    env = dict(os.environ, TQ_TEST_MAX_GRID_X="16", TQ_LIBRARY_PATH=build.FOLD_TEST_LIB)
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_gpu_norm.py::test_forward_and_backward",
           "tests/test_gpu_i8.py::test_cast", "tests/test_gpu_i8.py::test_product", "tests/test_gpu_i8.py::test_linear_is_cast_and_product",
           "tests/test_gpu_orth.py::test_the_steps", "tests/test_gpu_orth.py::test_update", "tests/test_gpu_orth.py::test_updates_of_many"]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
