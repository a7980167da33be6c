"""8-bit products in every kind of tile, with remainders, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2402_01798_amd import binding as B
from layer_common import TYPES, strided
from shape_sizes import I8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("m, n, k", [s for sizes in I8.values() for s in sizes])
def test_8_bit_product(m, n, k, dtype):
    """The sums, whole numbers below 2^53, are exact in 64 bits; three binary32 operations and a rounding, each as the library's."""
    g = np.random.default_rng(m + n + k)
    forms = []
    for rows in (m, n):
        codes = np.zeros((rows, -(-k // 128) * 128), dtype=np.int8)
        codes[:, :k] = g.integers(-128, 128, (rows, k))
        forms.append((torch.from_numpy(codes).cuda(), torch.from_numpy(np.exp(g.normal(size=rows) - 4).astype(np.float32)).cuda()))
    (a, sa), (b, sb) = forms
    bias = torch.from_numpy(g.normal(size=n).astype(np.float32)).cuda()
    nbytes = B.i8_matmul_workspace_bytes(m, n, k)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None
    out = strided(torch.zeros(m, n, dtype=TYPES[dtype]), 3, 1)
    B.tq_i8_matmul(B.I8Matrix(a, sa, m, k), B.I8Matrix(b, sb, n, k), out, ws, bias)
    want = (a.double() @ b.double().t().contiguous()).float() * sa.view(-1, 1) * sb + bias
    assert torch.equal(out, want.to(TYPES[dtype]))
    assert torch.as_strided(out, (m - 1, 3), out.stride(), out.storage_offset() + n).isnan().all()
