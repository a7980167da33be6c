"""The backward pass of layer norm on rows whose mean is far above their deviations, and on rows without any: every kernel, columns that fill what a
workgroup holds and columns that do not.  Against 64 bits, with tolerances counted from the roundings (layer_common)."""
import pytest
import torch

from paper_2402_01798_amd import binding as B
from layer_common import HALF_ULP, TYPES, U, norm_backward, norm_backward_bounds, norm_forward, norm_sums, strided

pytestmark = pytest.mark.gpu

# rows x columns of every kernel of the backward pass: a wavefront a row (of 16-bit types up to 1024 columns where there are many rows), 2, 4, 8, 16
# of them, rows over 16384 columns, rows over 32768
SHAPES = [(5, 1), (5, 64), (5, 500), (5, 512), (8200, 700), (5, 600), (5, 1000), (5, 1024), (5, 2001), (5, 3000), (5, 4096), (5, 8000), (5, 16001), (5, 16384),
          (70, 17003), (5, 32768), (5, 33001)]


def backward(x, dy, w, stats, dx=True):
    rows, cols = x.shape
    dx = torch.full_like(x, 7.0) if dx is True else dx
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(B.layernorm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda").fill_(255)
    B.tq_layernorm_backward(x, dy, w, stats, dx, dw, db, ws)
    return dx, dw, db


def statistics(x, w, eps):
    stats = torch.empty(x.shape[0], 2, device="cuda")
    B.tq_layernorm_forward(x, w, None, torch.empty_like(x), stats, eps)
    return stats


def rows_in_turn(rows, cols):
    """At least as many additions as a column's sum goes through: its part's rows, the parts of a thread, 32 threads."""
    parts = B.layernorm_workspace_bytes(rows, cols) // (8 * cols)
    return -(-rows // parts) + -(-parts // 32) + 40


@pytest.mark.parametrize("rows, cols", SHAPES)
@pytest.mark.parametrize("dtype, value, eps", [("f32", 1e37, 1e-5), ("f32", -(2.0 ** 121), 1e-5), ("f32", 1e24, 1e-30), ("f32", 0.1, 1e-30), ("bf16", 2.0 ** 121, 1e-5),
                                               ("bf16", 2.0 ** 79, 1e-30), ("f16", 60000.0, 1e-30)])
def test_equal_elements(rows, cols, dtype, value, eps):
    """h = 0 and 1 / deviation = eps^-1/2, so dx = (g - mean(g)) eps^-1/2 and nothing in dweight; a row in between that has deviations.
    mean(g) is off by the additions of its sum, a difference and two products of each element are rounded."""
    g = torch.Generator().manual_seed(cols)
    x = torch.full((rows, cols), value).to(TYPES[dtype])
    other = rows // 2
    x[other] = torch.randn(cols, generator=g).to(TYPES[dtype])
    dy = torch.randn(rows, cols, generator=g) * (1e-12 if dtype == "f16" else 0.1)
    dy = dy.to(TYPES[dtype])
    w = 1 + 0.3 * torch.randn(cols, generator=g)
    x, dy, w = x.cuda(), dy.cuda(), w.cuda()
    dx, dw, db = backward(x, dy, w, statistics(x, w, eps))
    eps32 = float(torch.tensor(eps, dtype=torch.float32))
    gw = dy.double() * w.double()
    r, mean = eps32 ** -0.5, gw.sum(dim=1, keepdim=True) / cols
    k = norm_sums(cols)
    want = r * (gw - mean)
    off = r * ((k + 6) * gw.abs().sum(dim=1, keepdim=True) / cols + 4 * gw.abs()) * U + 4 * U * want.abs()
    off = off + HALF_ULP[dtype] * (want.abs() + off) + {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}[dtype]
    equal = [i for i in range(rows) if i != other]
    assert ((dx.double() - want).abs() <= off)[equal].all()
    assert dx[other].isfinite().all()
    _, h, mean, _ = norm_forward(x[other:other + 1].double(), None, None, eps32)
    off = (dy[other].double().abs() * ((k / 2 + 8) * h[0].abs() + k + 6) * U if cols > 1 else torch.zeros(1, device="cuda", dtype=torch.float64))
    if cols > 1:                                            # of one column: equal too
        assert ((dw.double() - dy[other].double() * h[0]).abs() <= off + 2.0 ** -149).all()
    turns = rows_in_turn(rows, cols)
    sums = dy.double().sum(dim=0)
    assert ((db.double() - sums).abs() <= (turns + 4) * U * dy.double().abs().sum(dim=0) + 2.0 ** -149).all()


@pytest.mark.parametrize("rows, cols", [s for s in SHAPES if s[1] > 1])
@pytest.mark.parametrize("dtype, mean", [("f32", 2.0 ** 10), ("f32", 1e5), ("f32", -3e5), ("bf16", 100.0), ("f16", 1000.0)])
def test_a_mean_far_above_the_deviations(rows, cols, dtype, mean):
    """The statistics hold the mean as one binary32 number, up to 2^-24 |mean| from what it is; dx and dweight are those of the mean itself.
    With d that difference over the deviation, at most 2^-5 here, h before its own mean is taken out is off by (k / 2 + 6) u (|h| + d), its mean by
    (k + 2) u (1 + d), for mean |h| <= 1, and the difference by u |h|: together less than the bounds' (k / 2 + 8) u |h| + k u and another 6 u."""
    g = torch.Generator().manual_seed(cols + 1)
    x = (torch.randn(rows, cols, generator=g) + mean * (1 + 0.01 * torch.rand(rows, 1, generator=g))).to(TYPES[dtype])
    dy = (torch.randn(rows, cols, generator=g) * 0.1).to(TYPES[dtype])
    w = 1 + 0.3 * torch.randn(cols, generator=g)
    X, DY, W = strided(x, 3, 1), strided(dy, 1, 0), w.cuda()
    dx, dw, db = backward(X, DY, W, statistics(X, W, 1e-5))
    x64, dy64, w64 = X.double(), DY.double(), W.double()
    _, h, m, r = norm_forward(x64, w64, None, 1e-5)
    assert float((m.abs() * r).max()) * U <= 2.0 ** -5
    want = norm_backward(dy64, h, w64, r)
    bounds = norm_backward_bounds(x64, dy64, h, w64, 3 / r, r, dtype, rows_in_turn(rows, cols))       # 2 * mean * r * u: another 6 u
    for name, got, t, far in zip(("dx", "dweight", "dbias"), (dx, dw, db), want, bounds):
        worst = ((got.double() - t).abs() / far).max()
        assert worst <= 1, (name, float(worst))


@pytest.mark.parametrize("cols", [40, 900, 5000, 16001, 17003, 32768, 33001])
def test_some_of_the_gradients_and_in_place(cols):
    """Whatever is asked for and wherever it goes, the same bits."""
    g = torch.Generator().manual_seed(cols)
    x = (torch.randn(300, cols, generator=g) + 5000.0).cuda()
    dy, w = torch.randn(300, cols, generator=g).cuda(), torch.randn(cols, generator=g).cuda()
    stats = statistics(x, w, 1e-5)
    dx, dw, db = backward(x, dy, w, stats)
    _, dw2, db2 = backward(x, dy, w, stats, None)
    assert torch.equal(dw2, dw) and torch.equal(db2, db)
    only = torch.empty_like(x)
    B.tq_layernorm_backward(x, dy, w, stats, only)
    assert torch.equal(only, dx)
    for place in ("x", "dy"):
        held = {"x": x.clone(), "dy": dy.clone()}
        got = backward(held["x"], held["dy"], w, stats, held[place])
        assert all(torch.equal(a, b) for a, b in zip(got, (dx, dw, db)))
