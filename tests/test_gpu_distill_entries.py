"""What the loss says where the teacher names an id more than once."""
import numpy as np
import pytest
import torch

import learn_common as LC
from paper_2402_01798_amd import binding as B

pytestmark = pytest.mark.gpu


def test_the_loss_is_a_sum_over_entries_and_the_gradient_its_gradient():
    """Against the same teacher with its entries joined: the loss differs by the entropy of the split, the gradient does not."""
    rows, vocab, tau = 6, 700, 2.0
    g = torch.Generator(device="cuda").manual_seed(3)
    z = 2 * torch.randn(rows, vocab, generator=g, device="cuda")
    z[0, 17] = 60.0                                         # q of 17 next to 1: the loss of two halves is next to -tau^2 ln 2
    joined_ids = torch.tensor([[17, 4, -1], [17, 4, 699], [0, -1, -1], [5, 6, 7], [699, 0, 1], [17, 18, 19]], device="cuda")
    joined_t = torch.randn(rows, 3, generator=g, device="cuda")
    joined_t[0, 1] = -200.0
    # an entry in two with half of the probability each: tau ln 2 less of the logit
    ids, t = joined_ids.repeat(1, 2), (joined_t - tau * np.log(2.0)).repeat(1, 2)
    grad = torch.ones(rows, device="cuda")
    got = []
    for i, v in ((joined_ids, joined_t), (ids, t)):
        loss, dz, stats = torch.empty(rows, device="cuda"), torch.empty_like(z), torch.empty(rows, 2, device="cuda")
        B.tq_distill(z, i.contiguous(), v.float().contiguous(), grad, loss, dz, tau)
        forward = torch.empty(rows, device="cuda")
        B.tq_distill_forward(z, i.contiguous(), v.float().contiguous(), forward, stats, tau)
        want = LC.distill(z.double().cpu().numpy(), i.cpu().numpy(), v.double().cpu().numpy(), tau, np.ones(rows))
        # a logit z / tau of 30 and 100 in 32 bits and a few units of exp and log; two of them meet in a term of the loss
        eps = (60.0 / tau + 200.0 / tau + 32) * 2.0 ** -21
        for kernel in (loss, forward):
            assert (np.abs(kernel.double().cpu().numpy() - want[0]) <= 2 * eps * tau * tau).all()
        assert (np.abs(dz.double().cpu().numpy() - want[2]) <= 2 * eps * tau).all()
        got.append((loss, dz))
    assert ((got[0][0] - got[1][0] - tau * tau * np.log(2.0)).abs() <= 4 * eps * tau * tau).all()
    assert ((got[0][1] - got[1][1]).abs() <= 4 * eps * tau).all()
    assert float(got[1][0][0]) < -2.7 and (got[0][0] >= -2 * eps * tau * tau).all()
