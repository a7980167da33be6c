"""Distillation of rows past 32 bits, each call on the whole, and rows in pieces, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import learn_common as LC
from paper_2402_01798_amd import binding as B

pytestmark = pytest.mark.gpu


def close(got, want, bound):
    got = got.double().cpu().numpy()
    assert (np.abs(got - want) <= bound).all(), np.abs(got - want).max()


@pytest.mark.parametrize("vocab", [131_001, 131_072])
def test_every_call_on_rows_past_32_bits(vocab):
    """5.2e9 logits, the last 4 rows as the kernels find them there."""
    rows, top, tau = 40_000, 16, 2.0
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    z[-4:] = (3 * torch.randn(4, vocab, generator=g, device="cuda")).bfloat16()
    kept = z[-4:].clone()
    ids = torch.randint(0, vocab, (rows, top), generator=g, device="cuda")
    ids[-1, 0], ids[-2, 1], ids[-3] = vocab - 1, -1, torch.arange(top, device="cuda")
    t, grad = torch.randn(rows, top, generator=g, device="cuda"), 0.5 + torch.rand(rows, generator=g, device="cuda")
    loss_w, stats_w, dz_w, q = LC.distill(kept.double().cpu().numpy(), ids[-4:].cpu().numpy(), t[-4:].double().cpu().numpy(), tau,
                                          grad[-4:].double().cpu().numpy())
    # logits in 32 bits a few roundings of their size, exp and log a few units, the sum one for every doubling of its length, one rounding
    eps = (float(kept.float().abs().max()) / tau + float(t[-4:].abs().max()) / tau + 32) * 2.0 ** -21
    gn = grad[-4:].double().cpu().numpy()[:, None]
    bound = eps * tau * gn * (2 * q + np.abs(dz_w) / (tau * gn)) + 1.001 * LC.HALF_ULP["bf16"] * np.abs(dz_w) + 1e-37
    loss, stats = torch.full((rows,), 123.0, device="cuda"), torch.full((rows, 2), 123.0, device="cuda")
    B.tq_distill_forward(z, ids, t, loss, stats, tau)
    close(loss[-4:], loss_w, 2 * eps * tau * tau)
    close(stats[-4:], stats_w, np.array([0.0, eps]))
    B.tq_distill_backward(z, ids, t, stats, grad, z, tau)
    close(z[-4:], dz_w, bound)
    z.zero_()
    z[-4:] = kept
    loss.fill_(123.0)
    B.tq_distill(z, ids, t, grad, loss, z, tau)
    close(loss[-4:], loss_w, 2 * eps * tau * tau)
    close(z[-4:], dz_w, bound)
    assert (z[:-4].float().sum(dim=1).abs() < 0.05).all()   # the gradient of a row has the sum 0, up to its elements' roundings


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 40_000, "bf16"), (5, 131_008, "bf16"), (3, 65_540, "f32"), (40, 70_000, "f16")])
def test_rows_in_pieces_write_what_one_workgroup_writes(rows, vocab, dtype):
    """Every row begins at a multiple of 16 bytes, so that the pieces of few rows and the whole of many have the same loose elements."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    z = torch.randn(rows, vocab, generator=g, device="cuda").to(LC.TYPES[dtype])
    assert vocab * z.element_size() % 16 == 0
    ids = torch.randint(0, vocab, (rows, 30), generator=g, device="cuda")
    ids[:, 7], ids[:, 8], ids[:, 9] = ids[:, 3], 0, vocab - 1
    t, grad = torch.randn(rows, 30, generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda")
    loss, stats = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    B.tq_distill_forward(z, ids, t, loss, stats)
    many = -(-1100 // rows)
    few = B.tq_distill_backward(z, ids, t, stats, grad, torch.full_like(z, 9.0))
    in_place = z.clone()
    B.tq_distill_backward(in_place, ids, t, stats, grad, in_place)
    again = [v.repeat(many, *[1] * (v.dim() - 1)) for v in (z, ids, t, stats, grad)]
    whole = B.tq_distill_backward(*again, torch.full_like(again[0], 9.0)).view(many, rows, vocab)
    assert torch.equal(few, in_place) and (whole == few).all()
