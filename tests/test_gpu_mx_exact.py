"""Products of 4-bit matrices whose sums are exact in 32 bits in any order: what the kernels return has to be equal, bit for bit."""
import pytest
import torch

import learn_common as LC
from paper_2402_01798_amd import binding as B

pytestmark = pytest.mark.gpu


def small(rows, cols, seed):
    codes, scales, values = LC.small_form(rows, cols, seed)
    return B.MxMatrix(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), rows, cols), torch.from_numpy(values).cuda()


def scratch(nbytes):
    return torch.full((nbytes,), 0xA5, dtype=torch.uint8, device="cuda") if nbytes else None


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(5, 37, 2000), (20, 8300, 640), (40, 100, 2000), (300, 200, 1999), (64, 64, 8192), (70, 130, 20001),
                                   (2056, 1000, 1999), (700, 1301, 300), (2047, 2040, 513), (1111, 8001, 130), (1037, 8192, 260),
                                   (2051, 2045, 300), (3713, 3701, 520)])
def test_the_addend_is_added_once(m, n, k, out):
    """Gradients accumulated over batches: an addend far larger than the product costs one rounding, whichever kernel the size takes;
    added to every partial sum on the way, it would cost one at each."""
    (a, va), (b, vb) = small(m, k, 1), small(n, k, 2)
    product = (va @ vb.t().contiguous()).float()            # exact
    g = torch.Generator(device="cuda").manual_seed(3)
    add = torch.randn(m, n + 3, generator=g, device="cuda")[:, 2:n + 2] * (2.0 ** 16 * float(product.abs().mean()))
    want = (product + add).to(LC.TYPES[out])
    ws = scratch(B.mx_matmul_workspace_bytes(m, n, k))
    wide = torch.full((m, n + 2), 7.0, dtype=LC.TYPES[out], device="cuda")
    B.tq_mx_matmul(a, b, wide[:, :n], ws, add=add)
    assert torch.equal(wide[:, :n], want) and (wide[:, n:] == 7).all()
    if out == "f32":
        place = add.contiguous()
        B.tq_mx_matmul(a, b, place, ws, add=place)
        assert torch.equal(place, want)


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,n,k", [(33, 32641, 300), (64, 32640, 513), (64, 32801, 1100), (50, 128256, 130)])
def test_product_of_few_rows_and_a_large_vocabulary(m, n, k, out):
    (a, va), (b, vb) = small(m, k, 1), small(n, k, 2)
    product = (va @ vb.t().contiguous()).float()
    add = torch.randn(m, n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    for extra in (None, add):
        wide = torch.full((m, n + 3), 5.0, dtype=LC.TYPES[out], device="cuda")
        B.tq_mx_matmul(a, b, wide[:, 1:n + 1], scratch(B.mx_matmul_workspace_bytes(m, n, k)), extra)
        assert torch.equal(wide[:, 1:n + 1], (product if extra is None else product + extra).to(LC.TYPES[out]))
        assert (wide[:, 0] == 5).all() and (wide[:, n + 1:] == 5).all()


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", LC.LONG_PRODUCTS)
def test_product_over_a_long_axis(m, n, k, out):
    """k over workgroups and a second launch that joins them, whatever the workspace held: no part is left out or comes twice."""
    (a, va), (b, vb) = small(m, k, 1), small(n, k, 2)
    product = (va @ vb.t().contiguous()).float()
    nbytes = B.mx_matmul_workspace_bytes(m, n, k)
    assert nbytes > 0
    add = torch.randn(m, n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    for extra in (None, add):
        want = (product if extra is None else product + extra).to(LC.TYPES[out])
        for fill in (0x00, 0xFF):                           # 0xFF: NaN
            ws = torch.full((nbytes,), fill, dtype=torch.uint8, device="cuda")
            got = B.tq_mx_matmul(a, b, torch.full((m, n + 2), 5.0, dtype=LC.TYPES[out], device="cuda")[:, 1:n + 1], ws, extra)
            assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,n,k", LC.LONG_LINEARS)
def test_linear_over_a_long_axis(m, n, k, dtype):
    """On both sides of what is cast in the product, up to all that LDS holds."""
    x = torch.from_numpy(LC.small_tokens(m, k, 1)).to(LC.TYPES[dtype]).cuda()
    w, vw = small(n, k, 2)
    want = (x.double() @ vw.t().contiguous()).float()
    got = B.tq_mx_linear(x, w, torch.empty(m, n, device="cuda"), scratch(B.mx_linear_workspace_bytes(m, n, k)))
    assert torch.equal(got, want)
