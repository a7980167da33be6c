"""Casts of matrices of 256 tiles of 128 x 128 and more, which go by tiles where a transpose is wanted, byte for byte against the
definition: types, roundings, forms, special values, rows that begin anywhere."""
import functools
import os
import subprocess
import sys

import pytest
import torch

import learn_common as LC
from paper_2402_01798_amd import binding as B

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KEY = 2 ** 33 + 11, 2, 2 ** 32 - 6


def new_form(rows, cols):
    f = B.alloc_mx(rows, cols)
    f.codes.fill_(0xA5)                                     # everything has to be written, padding included
    f.scales.fill_(0xA5)
    return f


@functools.lru_cache(maxsize=2)
def case(rows, cols, dtype, stochastic):
    """The matrix, as a part of a wider one, and its two forms."""
    x = LC.hard_matrix(rows, cols + 9, dtype, rows + cols)
    r = LC.draws_of_all(rows, cols, *KEY) if stochastic else None
    v = x[:, 3:3 + cols].double().numpy()
    return x.cuda(), LC.mx_form_of_all(v, r), LC.mx_form_of_all(v.T, None if r is None else r.T)


def check(rows, cols, dtype, stochastic, forms):
    x, along, down = case(rows, cols, dtype, stochastic)
    f = new_form(rows, cols) if "r" in forms else None
    ft = new_form(cols, rows) if "c" in forms else None
    for part in (x[:, 3:3 + cols], x[:, 3:3 + cols].contiguous()):
        B.tq_mx_quantize(part, f, ft, B.MX_STOCHASTIC if stochastic else B.MX_NEAREST, *KEY)
        for form, want in ((f, along), (ft, down)):
            if form is not None:
                assert torch.equal(form.scales.cpu(), torch.from_numpy(want[1])) and torch.equal(form.codes.cpu(), torch.from_numpy(want[0]))
                form.codes.fill_(0x5A)
                form.scales.fill_(0x5A)


@pytest.mark.parametrize("rows,cols", [(3, 32700), (32700, 5), (2047, 2049), (2048, 1927)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("forms", ["c", "rc"])
def test_cast_in_tiles(rows, cols, dtype, stochastic, forms):
    assert -(-rows // 128) * -(-cols // 128) >= 256
    check(rows, cols, dtype, stochastic, forms)


@pytest.mark.parametrize("rows,cols", [(40, 160), (130, 35), (255, 1025)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("forms", ["r", "c", "rc"])
def test_cast_of_smaller_matrices(rows, cols, dtype, stochastic, forms):
    check(rows, cols, dtype, stochastic, forms)


def test_with_a_folded_grid():
    """Launches beyond one grid dimension are folded; a child process lowers the fold point and casts in tiles again."""
    from paper_2402_01798_amd import build
    assert os.path.exists(build.FOLD_TEST_LIB), "build it first: python -m paper_2402_01798_amd.build"
    env = dict(os.environ, TQ_TEST_MAX_GRID_X="40", TQ_LIBRARY_PATH=build.FOLD_TEST_LIB)
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_gpu_mx_cast_tiles.py::test_cast_in_tiles",
           "-k", "32700"]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]


@pytest.mark.parametrize("stochastic", [False, True])
def test_cast_in_tiles_past_32_bits(stochastic):
    """4.6e9 elements: the last rows and columns of both forms, with draws that count from the matrix's beginning."""
    rows, cols = 70_000, 65_664                             # cols: 513 groups of 128
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    first_row, first_col = rows // 128 * 128, cols - 128
    x[first_row:] = LC.hard_matrix(rows - first_row, cols, "bf16", 1).cuda()
    x[:, first_col:] = LC.hard_matrix(rows, 128, "bf16", 2).cuda()
    f, ft = B.alloc_mx(rows, cols), B.alloc_mx(cols, rows)
    B.tq_mx_quantize(x, f, ft, B.MX_STOCHASTIC if stochastic else B.MX_NEAREST, *KEY)
    corner = x[first_row:, first_col:].double().cpu().numpy()
    r = LC.draws_of_all(*corner.shape, *KEY, first_row=first_row, first_col=first_col) if stochastic else None
    codes, scales = LC.mx_form_of_all(corner, r)
    assert torch.equal(f.codes[first_row:, -64:].cpu(), torch.from_numpy(codes)) and torch.equal(f.scales[-1:, first_row:].cpu(), torch.from_numpy(scales))
    codes, scales = LC.mx_form_of_all(corner.T, None if r is None else r.T)
    assert torch.equal(ft.codes[first_col:, -64:].cpu(), torch.from_numpy(codes)) and torch.equal(ft.scales[-1:, first_col:].cpu(), torch.from_numpy(scales))
    kept = f.codes[first_row:].clone(), f.scales[:, first_row:].clone()
    B.tq_mx_quantize(x, f, None, B.MX_STOCHASTIC if stochastic else B.MX_NEAREST, *KEY)      # by rows: the same
    assert torch.equal(f.codes[first_row:], kept[0]) and torch.equal(f.scales[:, first_row:], kept[1])
