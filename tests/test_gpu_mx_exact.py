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
