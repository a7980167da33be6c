"""Layer norm against a plain 64-bit statement, with tolerances counted from the roundings (layer_common)."""
import pytest
import torch

from paper_2402_01798_amd import binding as B
from layer_common import TYPES, norm_backward, norm_backward_bounds, norm_forward, norm_forward_bound, strided

pytestmark = pytest.mark.gpu


def make(rows, cols, dtype, seed, mean=0.5, size=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, cols, generator=g) * torch.exp(0.5 * torch.randn(rows, 1, generator=g)) * size
         + mean * torch.randn(rows, 1, generator=g)).to(TYPES[dtype])
    dy = (torch.randn(rows, cols, generator=g) * 0.1).to(TYPES[dtype])
    return x, dy, 1 + 0.3 * torch.randn(cols, generator=g), 0.2 * torch.randn(cols, generator=g)


def rows_in_turn(rows, cols):
    """At least as many additions as a column's sum goes through: its part's rows, the parts of a thread, 32 threads."""
    parts = B.layernorm_workspace_bytes(rows, cols) // (8 * cols)
    return -(-rows // parts) + -(-parts // 32) + 40


def check(x, dy, w, b, dtype, eps=1e-5, extra=0, offset=0):
    rows, cols = x.shape
    X, DY = strided(x, extra, offset), strided(dy, extra + 1, offset)
    wd, bd = (None if t is None else t.cuda() for t in (w, b))
    y, dx = strided(torch.zeros_like(x), extra, offset), strided(torch.zeros_like(x), extra + 2, 0)
    stats, dw, db = (torch.empty(*s, device="cuda") for s in ((rows, 2), (cols,), (cols,)))
    ws = torch.empty(B.layernorm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.tq_layernorm_forward(X, wd, bd, y, stats, eps)
    B.tq_layernorm_backward(X, DY, wd, stats, dx, dw, db, ws)
    x64, dy64 = x.double().cuda(), dy.double().cuda()
    w64, b64 = (None if t is None else t.double() for t in (wd, bd))
    want, h, mean, r = norm_forward(x64, w64, b64, eps)
    assert ((y.double() - want).abs() <= norm_forward_bound(want, h, w64, b64, cols, dtype)).all()
    assert torch.allclose(stats[:, 0].double(), mean[:, 0], rtol=1e-6, atol=1e-5 * float(x64.abs().mean()))
    assert torch.allclose(stats[:, 1].double(), r[:, 0], rtol=1e-5)
    want = norm_backward(dy64, h, w64, r)
    bounds = norm_backward_bounds(x64, dy64, h, w64, mean, r, dtype, rows_in_turn(rows, cols))
    for name, got, t, far in zip(("dx", "dweight", "dbias"), (dx, dw, db), want, bounds):
        worst = ((got.double() - t).abs() / far).max()
        assert worst <= 1, (name, float(worst))
    if extra:                                                # what lies between the rows is left alone
        for t in (X, y, DY, dx):
            assert torch.as_strided(t, (rows - 1, t.stride(0) - cols), t.stride(), t.storage_offset() + cols).isnan().all()


SHAPES = [(1, 1), (3, 1), (2, 2), (5, 7), (1, 8), (9, 9), (64, 64), (33, 511), (7, 512), (6, 513), (10, 1001), (5, 1024), (3, 1025),
          (2, 2047), (5, 2049), (3, 4096), (4, 4099), (2, 8192), (3, 8200), (2, 16384), (3, 16385), (70, 20003), (2, 32768), (3, 32769), (2, 40001), (2500, 40), (1300, 130)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_forward_and_backward(rows, cols, dtype):
    x, dy, w, b = make(rows, cols, dtype, rows * 7 + cols)
    check(x, dy, w, b, dtype)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("cols", [5, 130, 1000, 3001, 9000, 17003])
def test_rows_apart_and_at_any_address(cols, dtype):
    x, dy, w, b = make(5, cols, dtype, cols)
    check(x, dy, w, b, dtype, extra=3, offset=1)


@pytest.mark.parametrize("wtype", ["bf16", "f16"])
@pytest.mark.parametrize("cols", [9, 700, 5000, 20000])
def test_weights_of_16_bits_or_none(cols, wtype):
    x, dy, w, b = make(4, cols, "bf16", cols)
    check(x, dy, w.to(TYPES[wtype]), b.to(TYPES[wtype]), "bf16")
    check(x, dy, None, b.to(TYPES[wtype]), "bf16")
    check(x, dy, w.to(TYPES[wtype]), None, "bf16")
    check(x, dy, None, None, "bf16")


@pytest.mark.parametrize("cols", [100, 1500, 6000, 18000])
def test_a_mean_far_above_the_deviations(cols):
    x, dy, w, b = make(4, cols, "f32", cols, mean=0.0)
    check(x + 1000.0, dy, w, b, "f32")


@pytest.mark.parametrize("cols", [64, 600, 3000, 17000])
@pytest.mark.parametrize("scale", [2.0 ** 120, 2.0 ** 70, 2.0 ** -40, 2.0 ** -120])
def test_the_ends_of_the_range(cols, scale):
    """Squares and sums outside binary32; only some of a workgroup's rows."""
    x, dy, w, b = make(6, cols, "f32", cols)
    x[1::2] *= scale
    y, stats = torch.empty(6, cols, device="cuda"), torch.empty(6, 2, device="cuda")
    B.tq_layernorm_forward(x.cuda(), w.cuda(), b.cuda(), y, stats, 1e-5)
    want, h, mean, r = norm_forward(x.double(), w.double(), b.double(), 1e-5)
    assert ((y.cpu().double() - want).abs() <= norm_forward_bound(want, h, w.double(), b.double(), cols, "f32")).all()
    assert torch.allclose(stats[:, 1].cpu().double(), r[:, 0], rtol=1e-5)
    dx = torch.empty(6, cols, device="cuda")
    B.tq_layernorm_backward(x.cuda(), dy.cuda(), w.cuda(), stats, dx)
    want = norm_backward(dy.double(), h, w.double(), r)[0]
    assert torch.allclose(dx.cpu().double(), want, rtol=1e-4, atol=1e-5 * float(want[0].abs().max()))


def test_the_largest_magnitudes():
    x = torch.full((3, 1000), 3e38)
    x[1, ::2] = -3e38
    x[2] = 1.0
    y = torch.empty(3, 1000, device="cuda")
    B.tq_layernorm_forward(x.cuda(), None, None, y, None, 1e-5)
    assert (y[0] == 0).all() and (y[2] == 0).all()
    assert torch.allclose(y[1].cpu(), torch.where(torch.arange(1000) % 2 == 0, -1.0, 1.0), atol=1e-5)


@pytest.mark.parametrize("cols", [9, 500, 3000, 17000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_nan_and_infinity_stay_in_their_row(cols, bad):
    x, dy, w, b = make(9, cols, "f32", cols)
    clean = torch.empty(9, cols, device="cuda")
    B.tq_layernorm_forward(x.cuda(), w.cuda(), b.cuda(), clean)
    x[4, cols // 2] = bad
    y, stats, dx = torch.empty_like(clean), torch.empty(9, 2, device="cuda"), torch.empty_like(clean)
    B.tq_layernorm_forward(x.cuda(), w.cuda(), b.cuda(), y, stats)
    B.tq_layernorm_backward(x.cuda(), dy.cuda(), w.cuda(), stats, dx)
    others = [0, 1, 2, 3, 5, 6, 7, 8]
    assert y[4].isnan().all() and stats[4, 1].isnan() and dx[4].isnan().all()
    assert torch.equal(y[others], clean[others]) and dx[others].isfinite().all()


def test_equal_elements():
    for cols in (1, 5, 700, 5000, 17000):
        x = torch.full((3, cols), 0.1, device="cuda")
        y = torch.empty_like(x)
        b = torch.arange(cols, device="cuda", dtype=torch.float32)
        B.tq_layernorm_forward(x, None, b, y, None, 1e-30)
        assert torch.equal(y, b.expand(3, cols))


@pytest.mark.parametrize("cols", [40, 900, 5000, 17000])
def test_in_place(cols):
    x, dy, w, b = (t.cuda() for t in make(5, cols, "bf16", cols))
    y, stats = torch.empty_like(x), torch.empty(5, 2, device="cuda")
    B.tq_layernorm_forward(x, w, b, y, stats)
    ws = torch.empty(B.layernorm_workspace_bytes(5, cols), dtype=torch.uint8, device="cuda")
    first = [torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")]
    B.tq_layernorm_backward(x, dy, w, stats, *first, ws)
    for target in ("dy", "x"):
        inputs = {"x": x.clone(), "dy": dy.clone()}
        again = [inputs[target], torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")]
        B.tq_layernorm_backward(inputs["x"], inputs["dy"], w, stats, *again, ws)
        assert all(torch.equal(a, f) for a, f in zip(again, first))
    z = x.clone()
    B.tq_layernorm_forward(z, w, b, z)
    assert torch.equal(z, y)


@pytest.mark.parametrize("cols", [40, 900, 5000, 17000])
def test_any_of_the_gradients_and_accumulation(cols):
    x, dy, w, b = (t.cuda() for t in make(300, cols, "f32", cols))
    y, stats = torch.empty_like(x), torch.empty(300, 2, device="cuda")
    B.tq_layernorm_forward(x, w, b, y, stats)
    ws = torch.empty(B.layernorm_workspace_bytes(300, cols), dtype=torch.uint8, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    B.tq_layernorm_backward(x, dy, w, stats, dx, dw, db, ws)
    only = torch.empty_like(x)
    B.tq_layernorm_backward(x, dy, w, stats, only)
    assert torch.equal(only, dx)
    for one, two in ((torch.empty_like(dw), None), (None, torch.empty_like(db))):
        B.tq_layernorm_backward(x, dy, w, stats, None, one, two, ws)
        assert one is None or torch.equal(one, dw)
        assert two is None or torch.equal(two, db)
    before = torch.randn(cols, device="cuda")
    more = [before.clone(), before.clone()]
    B.tq_layernorm_backward(x, dy, w, stats, dx, *more, ws, accumulate=True)
    assert torch.equal(more[0], before + dw) and torch.equal(more[1], before + db)


@pytest.mark.parametrize("cols", [6, 1100, 17000])
def test_gradients_against_differences(cols):
    """Central differences of the definition in 64 bits: off by the step's square."""
    x, dy, w, b = make(3, cols, "f32", cols + 1)
    x64, dy64, w64, b64 = (t.double() for t in (x, dy, w, b))
    stats, y = torch.empty(3, 2, device="cuda"), torch.empty(3, cols, device="cuda")
    B.tq_layernorm_forward(x.cuda(), w.cuda(), b.cuda(), y, stats)
    ws = torch.empty(B.layernorm_workspace_bytes(3, cols), dtype=torch.uint8, device="cuda")
    got = [torch.empty(3, cols, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")]
    B.tq_layernorm_backward(x.cuda(), dy.cuda(), w.cuda(), stats, *got, ws)
    loss = lambda x, w, b: float((norm_forward(x, w, b, 1e-5)[0] * dy64).sum())
    g = torch.Generator().manual_seed(1)
    for k, t in enumerate((x64, w64, b64)):
        way = torch.randn(t.shape, generator=g, dtype=torch.float64) * 1e-4
        args = [x64, w64, b64]
        plus, minus = args[:k] + [t + way] + args[k + 1:], args[:k] + [t - way] + args[k + 1:]
        slope = (loss(*plus) - loss(*minus)) / 2
        assert abs(float((got[k].cpu().double() * way).sum()) - slope) <= 1e-5 * float((got[k].cpu().double() * way).abs().sum())


def test_the_same_bits_every_time():
    x, dy, w, b = (t.cuda() for t in make(3000, 777, "bf16", 5))
    y, stats = torch.empty_like(x), torch.empty(3000, 2, device="cuda")
    ws = torch.empty(B.layernorm_workspace_bytes(3000, 777), dtype=torch.uint8, device="cuda")
    results = []
    for _ in range(3):
        B.tq_layernorm_forward(x, w, b, y, stats)
        got = [torch.empty_like(x), torch.empty(777, device="cuda"), torch.empty(777, device="cuda")]
        ws.fill_(255)
        B.tq_layernorm_backward(x, dy, w, stats, *got, ws)
        results.append([y.clone(), *got])
    for again in results[1:]:
        assert all(torch.equal(a, f) for a, f in zip(again, results[0]))
