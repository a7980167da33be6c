"""Random numbers of the example that runs everything: no two roundings share them."""
import os
import sys

import pytest

from paper_2402_01798_amd import binding as B

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_no_two_roundings_of_a_student_share_their_draws(monkeypatch):
    """A cast and a payload, or two casts, of one (seed, worker, step) would draw the same numbers: each triple occurs once."""
    import distill_student as D
    used = []
    quantize, compress = B.tq_mx_quantize, B.tq_compress_multi

    def record_quantize(x, form, form_t=None, rounding=B.MX_NEAREST, seed=0, worker=0, step=0):
        if rounding == B.MX_STOCHASTIC:
            used.append((seed, worker, step))
        return quantize(x, form, form_t, rounding, seed, worker, step)

    def record_compress(grads, params, payloads, bits, seed, first_worker, step, **kw):
        used.extend((seed, first_worker + i, step) for i in range(len(grads)))
        return compress(grads, params, payloads, bits, seed, first_worker, step, **kw)

    monkeypatch.setattr(B, "tq_mx_quantize", record_quantize)
    monkeypatch.setattr(B, "tq_compress_multi", record_compress)
    D.train(4)
    assert len(used) == 4 * 3 * D.WORKERS                   # two gradients cast and one compressed, of each worker
    assert len(set(used)) == len(used)
