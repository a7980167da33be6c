"""Distillation from a teacher's top logits (tq_distill.h) against the definition in 64 bits and against differences."""
import numpy as np
import pytest
import torch

import learn_common as LC
from paper_2402_01798_amd import binding as B

pytestmark = pytest.mark.gpu


def make(rows, vocab, top, dtype, seed, wide=False, spread=4.0):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy(rng.standard_normal((rows, vocab)) * spread).to(LC.TYPES[dtype])
    ids = rng.integers(0, vocab, (rows, top))
    ids[rng.random((rows, top)) < 0.1] = -1
    ids[rng.random((rows, top)) < 0.05] = vocab
    t = (rng.standard_normal((rows, top)) * 3).astype(np.float32)
    grad = rng.random(rows).astype(np.float32)
    grad[2::7] = 0
    if rows > 3:
        ids[3] = -1
    ids = torch.from_numpy(ids.astype(np.int64 if wide else np.int32))
    return z.cuda(), ids.cuda(), torch.from_numpy(t).cuda(), torch.from_numpy(grad).cuda()


def close(got, want, bound):
    got, want = got.double().cpu().numpy(), want.astype(np.float32).astype(np.float64)
    ok = (np.abs(got - want) <= bound) | (got == want) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), (np.argwhere(~ok)[:5], got[~ok][:5], want[~ok][:5])


def check(z, ids, t, grad, tau, dtype, in_place=False):
    rows, vocab = z.shape
    zn, idn, tn, gn = z.double().cpu().numpy(), ids.cpu().numpy(), t.double().cpu().numpy(), grad.double().cpu().numpy()
    loss_w, stats_w, dz_w, q = LC.distill(zn, idn, tn, tau, gn)
    # Every logit enters as z / tau in 32 bits, a few roundings of its size; exp and log add a few units, the row's sum one
    # for every doubling of its length.
    finite = np.where(np.abs(zn) < 1e4, np.abs(zn), 0).max() / tau + np.where(np.abs(tn) < 1e4, np.abs(tn), 0).max() / tau + 32
    eps = finite * 2.0 ** -21
    new = lambda: torch.full((rows,), 123.0, device="cuda")
    loss, stats = new(), torch.full((rows, 2), 123.0, device="cuda")
    B.tq_distill_forward(z, ids, t, loss, stats, tau)
    close(loss, loss_w, 2 * eps * tau * tau)
    close(stats, stats_w, np.array([0.0, eps]))
    # q and the teacher's share are each off by eps of themselves (where they cancel that is more than eps of the difference), and
    # the result is rounded once
    share = np.abs(dz_w) / np.maximum(tau * np.abs(gn)[:, None], 1e-30) + q
    dz_bound = eps * tau * np.abs(gn)[:, None] * (q + share) + 1.001 * LC.HALF_ULP[dtype] * np.abs(dz_w) \
        + (2.0 ** -25 if dtype == "f16" else 1e-37)
    zs = z.clone() if in_place else z
    dz = zs if in_place else torch.full_like(z, 55.0)
    B.tq_distill_backward(zs, ids, t, stats, grad, dz, tau)
    close(dz, dz_w, dz_bound)
    zs = z.clone() if in_place else z
    dz, loss = zs if in_place else torch.full_like(z, 55.0), new()
    B.tq_distill(zs, ids, t, grad, loss, dz, tau)
    close(loss, loss_w, 2 * eps * tau * tau)
    close(dz, dz_w, dz_bound)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows,vocab,top,tau", [(1, 1, 1, 1.0), (5, 7, 3, 2.0), (9, 64, 17, 0.5), (4, 1000, 64, 1.0), (6, 1027, 300, 4.0),
                                                (3, 8192, 8, 2.0), (5, 20001, 1024, 1.0), (2, 50257, 100, 3.0), (2, 131001, 128, 2.0),
                                                (1, 200003, 50, 1.0)])
def test_loss_and_gradient(dtype, in_place, rows, vocab, top, tau):
    check(*make(rows, vocab, top, dtype, rows * 31 + vocab, wide=bool(rows & 1)), tau, dtype, in_place)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,width", [(0, 512), (1, 509), (8, 500), (5, 513)])
def test_rows_of_a_wider_tensor(dtype, offset, width):
    z, ids, t, grad = make(6, 520, 20, dtype, 3)
    part = z[:, offset:offset + width]
    check(part, ids, t, grad, 1.0, dtype)
    wide = torch.full_like(z, 9.0)
    B.tq_distill(part, ids, t, grad, torch.empty(6, device="cuda"), wide[:, offset:offset + width])
    assert (wide[:, :offset] == 9).all() and (wide[:, offset + width:] == 9).all()


def test_ids_that_occur_twice():
    z, ids, t, grad = make(8, 300, 40, "f32", 5)
    ids[:, 20:] = ids[:, :20]
    ids[1] = 17
    check(z, ids, t, grad, 1.0, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [50, 5003])
def test_masked_logits(dtype, vocab):
    """-inf and the type's lowest value among the student's logits, whole rows of them, -inf among the teacher's."""
    z, ids, t, grad = make(12, vocab, 10, dtype, 8)
    grad += 0.25
    lowest = torch.finfo(z.dtype).min
    ids[:] = torch.arange(10, device="cuda") * (vocab // 20)
    z[0, vocab // 2:] = -float("inf")
    z[1, vocab // 2:] = lowest
    z[2] = -float("inf")                                    # nothing left: q = 0 everywhere
    z[3] = lowest
    z[4] = -float("inf")
    z[4, vocab - 1] = 1.0                                   # one left, which the teacher does not name
    z[5] = -float("inf")
    z[5, 0] = -3.0                                          # one left, which it does
    t[6, 3:] = -float("inf")
    t[7] = -float("inf")                                    # a teacher without anything
    t[8] = torch.finfo(torch.float32).min
    t[9, 1:] = torch.finfo(torch.float32).min
    z[10, :-1] = -float("inf")
    ids[10] = -1
    check(z, ids, t, grad, 2.0, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_and_infinity_stay_in_their_rows(dtype):
    z, ids, t, grad = make(9, 700, 6, dtype, 10)
    ids[:] = torch.arange(6, device="cuda") * 100
    grad += 0.5
    z[1, 650] = float("nan")
    z[2, 650] = float("inf")
    t[4, 2] = float("nan")
    t[5, 2] = float("inf")
    z[6, 3] = float("nan")
    ids[6] = -1                                             # no teacher: 0 whatever the logits
    z[7, 3] = float("nan")
    grad[7] = 0                                             # does not count: gradient 0
    t[8, 1], ids[8, 1] = float("nan"), -1                   # an absent entry's logit is not read
    loss, stats, dz, dz2 = torch.empty(9, device="cuda"), torch.empty(9, 2, device="cuda"), torch.empty_like(z), torch.empty_like(z)
    B.tq_distill_forward(z, ids, t, loss, stats)
    B.tq_distill_backward(z, ids, t, stats, grad, dz)
    loss2 = torch.empty(9, device="cuda")
    B.tq_distill(z, ids, t, grad, loss2, dz2)
    for n, d in ((loss, dz), (loss2, dz2)):
        assert torch.isnan(n).cpu().tolist() == [False, True, True, False, True, True, False, True, False]
        assert torch.isnan(d).all(dim=1).cpu().tolist() == [False, True, True, False, True, True, False, False, False]
        assert torch.isfinite(d[[0, 3, 6, 7, 8]]).all()
        assert (d[6] == 0).all() and (d[7] == 0).all() and n[6] == 0


def test_nan_beside_nothing_but_masked_logits():
    z, ids, t, grad = make(3, 3000, 6, "f32", 11)
    ids[:] = torch.arange(6, device="cuda") * 100
    grad += 0.5
    z[1:] = -float("inf")
    z[1, 2222] = float("nan")
    loss, dz = torch.empty(3, device="cuda"), torch.empty_like(z)
    B.tq_distill(z, ids, t, grad, loss, dz)
    assert torch.isnan(dz).all(dim=1).cpu().tolist() == [False, True, False] and torch.isnan(loss[1]) and torch.isinf(loss[2])


def test_gradient_against_differences_of_the_loss():
    """Central differences of the definition in 64 bits, and of the kernel's own loss."""
    z, ids, t, grad = make(5, 90, 12, "f32", 21, spread=1.5)
    grad[:] = 1.0
    tau, h = 1.5, 2.0 ** -7
    loss, dz = torch.empty(5, device="cuda"), torch.empty_like(z)
    B.tq_distill(z, ids, t, grad, loss, dz, tau)
    zn, idn, tn = z.double().cpu().numpy(), ids.cpu().numpy(), t.double().cpu().numpy()
    got = dz.double().cpu().numpy()
    up_l, down_l, stats = torch.empty(5, device="cuda"), torch.empty(5, device="cuda"), torch.empty(5, 2, device="cuda")
    for j in list(range(0, 90, 13)) + [int(i) for i in idn[0] if 0 <= i < 90][:3]:
        up, down = zn.copy(), zn.copy()
        up[:, j] += h
        down[:, j] -= h
        want = (LC.distill(up, idn, tn, tau)[0] - LC.distill(down, idn, tn, tau)[0]) / (2 * h)
        # the third derivative of tau^2 lse(z / tau) is at most 1 / tau
        assert (np.abs(got[:, j] - want) <= h * h / (6 * tau) + 1e-5).all()
        B.tq_distill_forward(torch.from_numpy(up).float().cuda(), ids, t, up_l, stats, tau)
        B.tq_distill_forward(torch.from_numpy(down).float().cuda(), ids, t, down_l, stats, tau)
        own = (up_l.double() - down_l.double()).cpu().numpy() / (2 * h)
        assert (np.abs(got[:, j] - own) <= h * h / (6 * tau) + 2 * 40 * 2.0 ** -21 * tau * tau / h).all()


def test_repeats_bit_for_bit():
    z, ids, t, grad = make(6, 30011, 200, "bf16", 30)
    out = []
    for _ in range(2):
        loss, dz = torch.empty(6, device="cuda"), torch.empty_like(z)
        B.tq_distill(z, ids, t, grad, loss, dz, 2.0)
        out.append((loss, dz))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


@pytest.mark.parametrize("top", [2, 3, 5, 37, 258, 1023])
def test_ids_that_occur_twice_among_any_number(top):
    z, ids, t, grad = make(7, 2048, top, "f32", 9)
    ids[:, top - 1] = ids[:, 0]                             # the first and the last
    ids[1] = 2047                                           # all of them
    ids[2, ::2] = int(ids[2, 0])
    ids[3, 1:] = -1                                         # those that are left out are not alike
    check(z, ids, t, grad, 2.0, "f32")
