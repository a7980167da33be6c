"""Newton-Schulz steps and the updates made of them against 64-bit arithmetic, with bounds that follow every rounding (layer_common)."""
import pytest
import torch

from paper_2402_01798_amd import binding as B
from layer_common import HALF_ULP, QUINTIC, TYPES, U, half, newton_schulz, newton_schulz_bound

pytestmark = pytest.mark.gpu

PRECISIONS = {"half": B.ORTH_HALF, "split": B.ORTH_SPLIT}
# what is held between products: a binary16 number, off by half a step; two of them, off by the second's half step, and the product of two
# second parts left out; sums of k terms in binary32, relative to the sum of magnitudes
UNIT = {"half": 2.0 ** -11, "split": 2.0 ** -21}


def matrix(rows, cols, seed, scale=1e-3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(0.5 * torch.randn(rows, cols, generator=g))
    return x * scale


def scratch(rows, cols, count, precision):
    ws = torch.empty(B.orthogonalize_workspace_bytes(rows, cols, count, PRECISIONS[precision]), dtype=torch.uint8, device="cuda")
    return ws.fill_(255)                                     # NaN wherever something is read that no kernel wrote


def bound(u, steps, precision, eps=1e-7):
    k = max(u.shape)
    return newton_schulz_bound(u, steps, eps, UNIT[precision], (k + 8) * U if precision == "split" else (k + 8) * U)


def check(g, precision, out="f32", steps=5, coefficients=None, eps=1e-7):
    rows, cols = g.shape
    got = torch.full((rows, cols), float("nan"), dtype=TYPES[out], device="cuda")
    B.tq_orthogonalize(g.cuda().contiguous(), got, scratch(rows, cols, 1, precision), steps=steps, precision=PRECISIONS[precision], eps=eps, coefficients=coefficients)
    used = coefficients or [QUINTIC] * steps
    u = g.double().cuda()
    want = newton_schulz(u, used, eps)
    far = bound(u, used, precision, eps) + HALF_ULP[out] * float(want.norm()) + U * float(want.norm())
    assert float((got.double() - want).norm()) <= far
    return got


SHAPES = [(1, 1), (1, 5), (5, 1), (1, 300), (2, 3), (7, 7), (17, 40), (40, 17), (32, 32), (33, 64), (63, 65), (64, 64), (64, 256), (100, 784), (784, 100),
          (128, 128), (129, 127), (130, 1000), (200, 200), (257, 300), (300, 257), (513, 640), (640, 513), (1000, 784)]


@pytest.mark.parametrize("precision", sorted(PRECISIONS))
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_the_steps(rows, cols, precision):
    check(matrix(rows, cols, rows + 3 * cols), precision)


@pytest.mark.parametrize("rows, cols", [(64, 256), (129, 127), (300, 257), (513, 640)])
def test_half_rounds_where_it_says(rows, cols):
    """One step against the same roundings in 64 bits.  A sum in binary32, off by some 2^-23 of itself, rounds to another binary16 number once
    in 2^-10 / 2^-23 / 2 = 2^12 times, which is then 2^-10 of it off: 2^-16 of the matrix for each of A and B, where a missing or added
    rounding makes 2^-11 / sqrt(3).  Over five steps such a test says nothing: a difference of 2^-16 changes one in 2^6 of the next
    roundings, which makes 2^-13, that one in 2^3 of those after it, and from then on the two round independently."""
    g = matrix(rows, cols, rows)
    got = torch.empty(rows, cols, device="cuda")
    B.tq_orthogonalize(g.cuda(), got, scratch(rows, cols, 1, "half"), steps=1, precision=B.ORTH_HALF)
    u = g.double().cuda()
    want = newton_schulz(u, [QUINTIC], 1e-7, half)
    assert float((got.double() - want).norm()) <= 2.0 ** -14 * float(want.norm())
    assert float((newton_schulz(u, [QUINTIC], 1e-7) - want).norm()) > 2.0 ** -13 * float(want.norm())


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("precision", sorted(PRECISIONS))
def test_types(dtype, precision):
    for rows, cols in ((70, 200), (200, 70)):
        g = matrix(rows, cols, 4, 0.1).to(TYPES[dtype])
        for out in TYPES:
            check(g, precision, out)


def test_default_precisions():
    g = matrix(60, 90, 1).cuda()
    for dtype, precision in ((torch.float32, "split"), (torch.bfloat16, "half"), (torch.float16, "half")):
        one, two = torch.empty(60, 90, dtype=dtype, device="cuda"), torch.empty(60, 90, dtype=dtype, device="cuda")
        B.tq_orthogonalize(g, one, scratch(60, 90, 1, "split"))
        B.tq_orthogonalize(g, two, scratch(60, 90, 1, precision), precision=PRECISIONS[precision])
        assert torch.equal(one, two)


@pytest.mark.parametrize("steps", [1, 2, 3, 16])
def test_numbers_of_steps(steps):
    """16 steps of the cubic 1.5 s - 0.5 s^3, which ends at singular values of 1: rows are orthonormal then."""
    cubic = [(1.5, -0.5, 0.0)] * steps
    g = torch.linalg.qr(matrix(150, 90, 3).double())[0].float() * torch.linspace(0.4, 1.0, 90)
    got = check(g, "split", steps=steps, coefficients=cubic)
    check(g.t().contiguous(), "split", steps=steps, coefficients=cubic)
    check(g, "half", steps=steps, coefficients=cubic)
    if steps < 4:                                            # the quintic's slope is up to 4: after 16 steps 4^16 * 2^-11 bounds nothing
        check(g, "half", steps=steps, coefficients=[QUINTIC] * steps)
    if steps == 16:
        one = got.double().t() @ got.double()
        assert float((one - torch.eye(90, device="cuda")).abs().max()) < 1e-4


def test_coefficients_of_each_step():
    table = [(3.4445, -4.775, 2.0315), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375), (1.5, -0.5, 0.0)]
    for shape in ((90, 40), (128, 300)):
        for precision in PRECISIONS:
            check(matrix(*shape, 9), precision, steps=4, coefficients=table)


@pytest.mark.parametrize("precision", sorted(PRECISIONS))
def test_sizes_of_numbers(precision):
    """The norm takes the size away: a power of two changes nothing (eps apart), zero stays zero, the smallest are as eps leaves them."""
    g = matrix(40, 70, 2, 1.0)
    results = []
    for scale in (2.0 ** 100, 1.0, 2.0 ** -60):
        results.append(check(g * scale, precision, eps=1e-30))
    assert torch.equal(results[0], results[1]) and torch.equal(results[1], results[2])
    check(g * 1e-30, precision)
    check(g * 3e37, precision)
    zero = torch.empty(40, 70, device="cuda")
    B.tq_orthogonalize(torch.zeros(40, 70, device="cuda"), zero, scratch(40, 70, 1, precision), precision=PRECISIONS[precision])
    assert (zero == 0).all()
    one = torch.zeros(40, 70)
    one[3, 5] = 5.0
    check(one, precision)
    rows = g.clone()
    rows[::3] = 0
    got = check(rows, precision)
    assert (got[::3] == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("shape", [(30, 50), (200, 150)])
def test_nan_and_infinity_spread(bad, shape):
    g = matrix(*shape, 1)
    g[7, 9] = bad
    for precision in PRECISIONS:
        out = torch.empty(*shape, device="cuda")
        B.tq_orthogonalize(g.cuda(), out, scratch(*shape, 1, precision), precision=PRECISIONS[precision])
        assert out.isnan().all()


def test_in_place_and_many_at_once():
    for shape in ((50, 90), (300, 140)):
        for precision in PRECISIONS:
            gs = [matrix(*shape, seed).bfloat16().cuda() for seed in range(5)]
            single = []
            for g in gs:
                out = torch.empty_like(g)
                single.append(B.tq_orthogonalize(g, out, scratch(*shape, 1, precision), precision=PRECISIONS[precision]))
            B.tq_orthogonalize_multi(gs, gs, scratch(*shape, 5, precision), precision=PRECISIONS[precision])
            assert all(torch.equal(a, b) for a, b in zip(gs, single))


def plain_update(g, v, theta, eta, momentum, nesterov, decay, scale, precision):
    """v' and theta' in 64 bits, and how far the library's may be from them."""
    g, v, theta = g.double().cuda(), v.double().cuda(), theta.double().cuda()
    new_v = momentum * v + g
    u = g + momentum * new_v if nesterov else new_v
    steps = [QUINTIC] * 5
    o = newton_schulz(u, steps, 1e-7)
    off_v = 2 * U * ((momentum * v).abs() + g.abs() + new_v.abs())
    # u's own rounding goes through the first step's normalisation and all slopes, as a unit of 4 u would
    off_o = newton_schulz_bound(u, steps, 1e-7, UNIT[precision] + 8 * U, (max(g.shape) + 8) * U)
    new_theta = theta - eta * (scale * o + decay * theta)
    off = abs(eta * scale) * off_o + 4 * U * float((theta.abs() + abs(eta) * (abs(scale) * o.abs() + abs(decay) * theta.abs())).norm())
    return new_v, off_v, new_theta, off


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows, cols, nesterov, precision", [(1, 1, True, "split"), (70, 33, True, "split"), (33, 70, False, "split"), (300, 784, True, "half"),
                                                             (784, 300, False, "half"), (129, 64, True, "split")])
def test_update(rows, cols, nesterov, precision, dtype):
    g = matrix(rows, cols, 1).to(TYPES[dtype])
    v, theta = matrix(rows, cols, 2, 1e-2), matrix(rows, cols, 3, 0.05)
    numbers = dict(eta=0.02, momentum=0.95, weight_decay=0.01, scale=1.5)
    V, T = v.cuda(), theta.cuda()
    new_v, new_t = torch.empty_like(V), torch.empty_like(T)
    ws = scratch(rows, cols, 1, precision)
    B.tq_orthogonal_update(g.cuda(), V, T, ws, nesterov=nesterov, precision=PRECISIONS[precision], velocity_out=new_v, theta_out=new_t, **numbers)
    f32 = {k: float(torch.tensor(x)) for k, x in numbers.items()}                  # as the call takes them
    want_v, off_v, want_t, off_t = plain_update(g, v, theta, f32["eta"], f32["momentum"], nesterov, f32["weight_decay"], f32["scale"], precision)
    assert ((new_v.double() - want_v).abs() <= off_v).all()
    assert float((new_t.double() - want_t).norm()) <= off_t
    assert torch.equal(V.cpu(), v) and torch.equal(T.cpu(), theta)
    B.tq_orthogonal_update(g.cuda(), V, T, ws, nesterov=nesterov, precision=PRECISIONS[precision], **numbers)
    assert torch.equal(V, new_v) and torch.equal(T, new_t)


def test_updates_of_many():
    shape = (96, 130)
    gs = [matrix(*shape, i).cuda() for i in range(4)]
    vs, ts = [matrix(*shape, 10 + i).cuda() for i in range(4)], [matrix(*shape, 20 + i).cuda() for i in range(4)]
    single = []
    for g, v, t in zip(gs, vs, ts):
        v, t = v.clone(), t.clone()
        B.tq_orthogonal_update(g, v, t, scratch(*shape, 1, "split"), eta=0.1)
        single.append((v, t))
    B.tq_orthogonal_update_multi(gs, vs, ts, scratch(*shape, 4, "split"), eta=0.1)
    assert all(torch.equal(v, a) and torch.equal(t, b) for v, t, (a, b) in zip(vs, ts, single))
