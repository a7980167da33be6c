"""Orthogonalised matrices and updates, small and in every kind of tile: as near to 64 bits as the roundings that the header names leave them."""
import pytest
import torch

from paper_2402_01798_amd import binding as B
from layer_common import HALF_ULP, QUINTIC, TYPES, U, half, newton_schulz, pair
from shape_sizes import ORTH

pytestmark = pytest.mark.gpu

PRECISIONS = {"half": B.ORTH_HALF, "split": B.ORTH_SPLIT}


def matrices(rows, cols, count, seed):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(rows, cols, generator=g) * torch.exp(0.5 * torch.randn(rows, cols, generator=g)) * 1e-3).cuda() for _ in range(count)]


def in_32_bits(u, steps, eps):
    """The steps by products in binary32."""
    flip = u.shape[0] > u.shape[1]
    x = (u / (torch.sqrt((u * u).sum()) + eps)).float()
    x = x.t().contiguous() if flip else x
    a, b, c = QUINTIC
    for _ in range(steps):
        gram = x @ x.t().contiguous()
        x = (a * torch.eye(x.shape[0], device=x.device) + b * gram + c * (gram @ gram)) @ x
    return (x.t().contiguous() if flip else x).double()


class Errors:
    """Norm and largest element of the differences of several matrices."""

    def __init__(self):
        self.square, self.largest = 0.0, 0.0

    def add(self, t):
        self.square += float((t * t).sum())
        self.largest = max(self.largest, float(t.abs().max()))

    @property
    def norm(self):
        return self.square ** 0.5


def references(us, steps, precision, eps=1e-7):
    """What 64 bits give, and errors that the stated roundings leave: of the same steps with the same things rounded; as pairs, whose sums are
    binary32 too, those of binary32 products beside them.  The library's roundings fall elsewhere, each with the same spread, so that over thousands
    of elements norm and largest element of its errors are much like these; they are allowed four times as much.  That is a long way below what a
    product of fewer bits, a row in a wrong place or a k left out makes."""
    wants, errors = [], [Errors(), Errors()]
    for u in us:
        u = u.double()
        want = newton_schulz(u, [QUINTIC] * steps, eps)
        wants.append(want)
        errors[0].add(newton_schulz(u, [QUINTIC] * steps, eps, half if precision == "half" else pair) - want)
        if precision == "split":
            errors[1].add(in_32_bits(u, steps, eps) - want)
    return wants, 4 * sum(e.norm for e in errors), 4 * sum(e.largest for e in errors)


def check(gots, wants, norm, largest, precision, by_element=True):
    off, size = Errors(), Errors()
    for got, want in zip(gots, wants):
        off.add(got.double() - want)
        size.add(want)
    assert norm <= {"half": 2.0 ** -6, "split": 2.0 ** -14}[precision] * size.norm, "the bound has to say something"
    floor = 2.0 ** -22                                       # of a result that no rounding happens to touch: the last products and sums in binary32
    assert off.norm <= norm + floor * size.norm, (off.norm / size.norm, norm / size.norm)
    if by_element:
        assert off.largest <= largest + floor * size.largest, (off.largest, largest)


def scratch(rows, cols, count, precision):
    ws = torch.empty(B.orthogonalize_workspace_bytes(rows, cols, count, PRECISIONS[precision]), dtype=torch.uint8, device="cuda")
    return ws.fill_(255)                                     # NaN wherever something is read that no kernel wrote


def run(gs, precision, steps=5, out=torch.float32):
    rows, cols = gs[0].shape
    outs = [torch.full((rows, cols), float("nan"), dtype=out, device="cuda") for _ in gs]
    B.tq_orthogonalize_multi(gs, outs, scratch(rows, cols, len(gs), precision), steps=steps, precision=PRECISIONS[precision])
    return outs


CASES = [(p, r, c, n) for p in sorted(ORTH) for r, c, n in ORTH[p]]


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("precision, r, c, count", CASES)
def test_orthogonalised_matrices(precision, r, c, count, turned):
    rows, cols = (c, r) if turned else (r, c)
    gs = matrices(rows, cols, count, r + c)
    check(run(gs, precision), *references(gs, 5, precision), precision)


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("precision, r, c, count", CASES)
def test_updates(precision, r, c, count, turned):
    """theta' = theta - O, with theta a hundredth of O's elements: O's own rounding is all there is."""
    rows, cols = (c, r) if turned else (r, c)
    dtype = torch.bfloat16 if precision == "half" else torch.float32
    gs = [g.to(dtype) for g in matrices(rows, cols, count, r + c + 1)]
    vs = matrices(rows, cols, count, r + c + 2)
    thetas = [t * (10.0 / max(rows, cols) ** 0.5) for t in matrices(rows, cols, count, r + c + 3)]
    new_vs, new_thetas = [torch.full_like(v, float("nan")) for v in vs], [torch.full_like(t, float("nan")) for t in thetas]
    B.tq_orthogonal_update_multi(gs, vs, thetas, scratch(rows, cols, count, precision), eta=1.0, momentum=0.5, precision=PRECISIONS[precision],
                                 velocities_out=new_vs, thetas_out=new_thetas)
    us = []
    for g, v, new in zip(gs, vs, new_vs):
        want = 0.5 * v + g.float()                           # half of v is exact: one rounding, as the library's
        assert torch.equal(new, want)
        us.append(g.float() + 0.5 * want)                    # likewise
    wants, norm, largest = references(us, 5, precision)
    check([t.double() - n.double() for t, n in zip(thetas, new_thetas)], wants, norm, largest + 2 * U * max(float(w.abs().max()) for w in wants), precision)


@pytest.mark.parametrize("precision", sorted(PRECISIONS))
@pytest.mark.parametrize("rows, cols", [(1, 1), (1, 5), (5, 1), (1, 300), (2, 3), (7, 7), (17, 40), (40, 17), (32, 32), (33, 64), (63, 65), (64, 64), (64, 256), (100, 784), (784, 100),
                                        (128, 128), (129, 127), (130, 1000), (200, 200), (257, 300), (300, 257), (513, 640), (640, 513), (1000, 784), (32, 900), (160, 128)])
def test_small_and_middling_matrices(rows, cols, precision):
    """As many at once as it takes for a few thousand elements, in up to three calls."""
    count = max(1, min(64, 8192 // (rows * cols)))
    for steps in (1, 2, 5):
        gs = matrices(rows, cols, count, rows + 3 * cols + steps)
        check(run(gs, precision, steps), *references(gs, steps, precision), precision, by_element=rows * cols * count >= 4096)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows, cols", [(64, 256), (300, 140), (784, 1000)])
def test_results_of_16_bits_as_pairs_lose_their_own_rounding_only(rows, cols, dtype):
    gs = [g.to(TYPES[dtype]) for g in matrices(rows, cols, 1, rows)]
    got = run(gs, "split", out=TYPES[dtype])[0].double()
    wants, norm, largest = references(gs, 5, "split")
    want = wants[0]
    assert ((got - want).abs() <= HALF_ULP[dtype] * (want.abs() + largest) + largest).all()
    rounded = want.to(TYPES[dtype]).double()
    # An element that is off by d rounds to another number, a step s away, in d / s of all cases: the squares of such differences sum up to the sum of
    # d s, at most |d| |s| in the norms: 4 * 2.6e-6 * 2^-10 of the square of the result's norm for 784 x 1000, fp16, where one more rounding to that type
    # would make the square of the rounding's norm, 3.6e-8 of it.
    off = Errors()
    off.add(got - rounded)
    far = norm * 2 * HALF_ULP[dtype] * float(want.norm())
    assert off.square <= far and far < float((rounded - want).norm()) ** 2


@pytest.mark.parametrize("rows, cols", [(64, 256), (300, 140), (784, 1000), (1024, 1024)])
def test_what_binary16_operands_cost(rows, cols):
    """As tq_orth.h says: more than the rounding of an fp16 result, less than that of a bf16 result."""
    gs = matrices(rows, cols, 1, rows + 1)
    want = references(gs, 5, "half")[0][0]
    off = float((run(gs, "half")[0].double() - want).norm() / want.norm())
    for dtype in ("bf16", "f16"):
        rounding = float((want.to(TYPES[dtype]).double() - want).norm() / want.norm())
        assert (off < rounding) == (dtype == "bf16")
