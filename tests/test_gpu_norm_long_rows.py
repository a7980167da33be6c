"""Layer norm of rows so long that a chain of binary32 additions would be seen: means far above the deviations, equal elements."""
import pytest
import torch

from paper_2402_01798_amd import binding as B
from layer_common import U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [32769, 1 << 20, (1 << 24) + 3, (1 << 26) + 1])
@pytest.mark.parametrize("value, eps", [(33000.0, 1e-5), (1000.3, 1e-30), (0.1, 1e-30), (-1.7e38, 1e-5)])
def test_equal_elements(cols, value, eps):
    x = torch.full((2, cols), value, device="cuda")
    y, stats = torch.empty_like(x), torch.empty(2, 2, device="cuda")
    B.tq_layernorm_forward(x, None, None, y, stats, eps)
    assert (y == 0).all()
    assert torch.equal(stats[:, 0], x[:, 0])
    dy = torch.zeros_like(x)
    dy[:, 0] = 1
    B.tq_layernorm_backward(x, dy, None, stats, dy)
    r = float(torch.tensor(eps)) ** -0.5                     # dx = (dy - 1 / cols) r
    assert torch.allclose(dy[:, 0].double(), torch.tensor(r * (1 - 1 / cols), dtype=torch.float64, device="cuda"), rtol=1e-6, atol=0)


@pytest.mark.parametrize("cols", [40001, 1 << 20, (1 << 24) + 3, (1 << 26) + 1])
@pytest.mark.parametrize("mean", [0.0, 1000.0])
def test_forward(cols, mean):
    """The sums are right to 2^-24 of themselves whatever the length: m + c, binary32 numbers both, is within 2^-24 of the deviation from the mean (of
    |x - m|, a few times the first mean's rounding), r and each product are rounded."""
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(1, cols, generator=g, device="cuda") + mean
    y, stats = torch.empty_like(x), torch.empty(1, 2, device="cuda")
    B.tq_layernorm_forward(x, None, None, y, stats, 1e-5)
    d = x.double()
    d -= d.mean()
    r = 1 / torch.sqrt((d * d).mean() + float(torch.tensor(1e-5)))
    assert abs(float(stats[0, 1]) / float(r) - 1) <= 4 * U
    assert abs(float(stats[0, 0]) - float(x.double().mean())) <= U * mean + 4 * U
    assert float(((d * r - y.double()).abs() - 8 * U * (d * r).abs()).max()) <= 4 * U


@pytest.mark.parametrize("cols", [40001, 1 << 20, (1 << 24) + 3, (1 << 26) + 1])
def test_backward(cols):
    """Gradients of one sign: their mean is the sum that a long chain would be off in.  h is off by 8 u of itself and 4 u (test_forward), the means by a
    rounding and by what h's error adds; each of the three differences and products is rounded."""
    g = torch.Generator(device="cuda").manual_seed(cols + 1)
    x = torch.randn(1, cols, generator=g, device="cuda") + 100.0
    dy = torch.rand(1, cols, generator=g, device="cuda") + 0.5
    stats, dx, dw = torch.empty(1, 2, device="cuda"), torch.empty_like(x), torch.empty(cols, device="cuda")
    B.tq_layernorm_forward(x, None, None, dx, stats, 1e-5)
    ws = torch.empty(B.layernorm_workspace_bytes(1, cols), dtype=torch.uint8, device="cuda")
    B.tq_layernorm_backward(x, dy, None, stats, dx, dw, None, ws)
    h = x.double()
    h -= h.mean()
    r = 1 / torch.sqrt((h * h).mean() + float(torch.tensor(1e-5)))
    h *= r
    assert float(((dy * h - dw).abs() - 9 * U * (dy * h).abs()).max()) <= 6 * U
    s1, s2 = dy.double().mean(), (dy * h).mean()
    want = r * (dy - s1 - h * s2)
    off = float(r) * U * (4 * (dy.double() + s1) + (h.abs() + 1) * (16 * s2.abs() + 16 * dy.double().mean()))
    assert ((dx - want).abs() <= off + 8 * U * want.abs()).all()
    again = dy.clone()
    dw2 = torch.empty_like(dw)
    B.tq_layernorm_backward(x, again, None, stats, again, dw2, None, ws)
    assert torch.equal(again, dx) and torch.equal(dw2, dw)
