"""The inputs of the exact product tests: sums that are exact in any order, and to which every group of 128 elements contributes, so
that a product which leaves one out is not equal.  A bound that grows with the number of terms would not see that: the sum of
k random terms grows with the square root of k alone."""
import numpy as np
import pytest

import learn_common as LC


def contributions(a, b):
    """[groups, m, n]: what each group of 128 elements of k adds to the product."""
    k = a.shape[1]
    pad = lambda v: np.pad(v, ((0, 0), (0, -k % 128))).reshape(v.shape[0], -1, 128).transpose(1, 0, 2)
    return pad(a) @ pad(b).transpose(0, 2, 1)


@pytest.mark.parametrize("linear", [False, True])
def test_no_group_can_be_left_out(linear):
    for m, n, k in LC.LONG_LINEARS if linear else LC.LONG_PRODUCTS:
        a = LC.small_tokens(m, k, 1) if linear else LC.small_form(m, k, 1)[2]
        b = LC.small_form(n, k, 2)[2]
        assert (np.abs(a) @ np.abs(b).T).max() * 4 <= 2 ** 24           # quarters: exact whatever the order
        parts = contributions(a, b)
        want = parts.sum(axis=0)
        assert (want != 0).mean() > 0.9
        short = k % 128 if k % 128 else 128                             # a last group of a few elements adds nothing more often
        for i, part in enumerate(parts):
            assert (part != 0).mean() > (0.5 if i < len(parts) - 1 or short > 8 else 0.2), (m, n, k, i)


def test_small_tokens_are_exact_in_4_bits():
    x = LC.small_tokens(3, 500, 1)
    x[0, :32] = 0.0
    x[1, :32] = 0.5
    codes, scales = LC.mx_form(x)
    assert (LC.mx_values(codes, scales, 500) == x).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (7, 31), (5, 128), (9, 300), (40, 136), (21, 1000)])
def test_all_blocks_at_a_time_is_block_by_block(rows, cols):
    key = 2 ** 40 + 7, 3, 2 ** 31 + 5
    x = LC.hard_matrix(rows, cols, "f32", rows).double().numpy()
    r = LC.draws(rows, cols, *key)
    assert (LC.draws_of_all(rows, cols, *key) == r).all()
    if rows > 4 and cols > 40:
        assert (LC.draws_of_all(rows - 3, cols - 16, *key, first_row=3, first_col=16) == r[3:, 16:]).all()
    for d in (None, r):
        for one, all_of_them in zip(LC.mx_form(x, d), LC.mx_form_of_all(x, d)):
            assert one.shape == all_of_them.shape and (one == all_of_them).all()
