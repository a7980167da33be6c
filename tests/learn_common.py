"""Plain 64-bit statements of the 4-bit matrix format and of distillation, written from their definitions (tq_mx.h,
tq_distill.h), for the tests of the kernels."""
import numpy as np
import torch

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # p bits of significand: 2^-p of a value in [1, 2)


def philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 on Python integers: four words."""
    m = 0xFFFFFFFF
    k0, k1 = seed & m, seed >> 32 & m
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = p1 >> 32 ^ c1 ^ k0, p1 & m, p0 >> 32 ^ c3 ^ k1, p0 & m
        k0, k1 = k0 + 0x9E3779B9 & m, k1 + 0xBB67AE85 & m
    return c0, c1, c2, c3


def draws(rows, cols, seed, worker, step):
    out = np.zeros((rows, -(-cols // 8) * 8), dtype=np.int64)
    for i in range(rows):
        for j in range(0, cols, 8):
            for w, word in enumerate(philox(j // 8, i, worker, step, seed)):
                out[i, j + 2 * w], out[i, j + 2 * w + 1] = word & 0xFFFF, word >> 16
    return out[:, :cols]


def mx_form(x, r=None):
    """(codes [rows, 64 G], scales [G, rows, 4]) of a float64 matrix that float32 holds; r = draws for stochastic rounding."""
    rows, cols = x.shape
    groups = -(-cols // 128)
    nibbles = np.zeros((rows, groups * 128), dtype=np.uint8)
    scales = np.zeros((groups, rows, 4), dtype=np.uint8)
    for i in range(rows):
        for j in range(0, cols, 32):
            v = x[i, j:j + 32]
            a = np.abs(v)
            if not np.isfinite(a).all():
                scales[j // 128, i, j // 32 % 4] = 255
                continue
            largest = a.max()
            if largest > 0:
                mantissa, e = np.frexp(largest)             # in [0.5, 1): largest = mantissa 2^e
                e = e - 3 + (1 if r is not None and mantissa > 0.75 else 0)
                byte = max(int(e) + 127, 0)
            else:
                byte = 0
            scales[j // 128, i, j // 32 % 4] = byte
            t = a * 2.0 ** (127 - byte)
            for n, tn in enumerate(t):
                low = int(np.searchsorted(GRID, min(tn, 6.0), side="right")) - 1
                if low == 7:
                    code = 7
                else:
                    share = (tn - GRID[low]) / (GRID[low + 1] - GRID[low])
                    if r is None:
                        up = share > 0.5 or (share == 0.5 and low % 2 == 1)
                    else:
                        up = int(np.floor(share * 65536)) + int(r[i, j + n]) >= 65536
                    code = low + up
                nibbles[i, j + n] = code + (8 if np.signbit(v[n]) else 0)
    return nibbles[:, 0::2] | nibbles[:, 1::2] << 4, scales


def mx_values(codes, scales, cols):
    rows = codes.shape[0]
    nibbles = np.stack([codes & 15, codes >> 4], axis=2).reshape(rows, -1)[:, :cols]
    s = scales.astype(np.float64).transpose(1, 0, 2).reshape(rows, -1)
    power = np.where(s == 255, np.nan, 2.0 ** (s - 127)).repeat(32, axis=1)[:, :cols]
    return np.where(nibbles >= 8, -1.0, 1.0) * GRID[nibbles & 7] * power


def product_bound(a, b, k, out, ref):
    """How far a product of exact terms may be off: k additions in 32 bits, each off by one unit at most, and the rounding."""
    return k * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T) + 1.001 * HALF_ULP[out] * np.abs(ref) + (2.0 ** -25 if out == "f16" else 0.0)


def distill(z, ids, t, tau, grad=None):
    """(loss, stats [rows, 2], dz, q) in float64, as tq_distill.h defines them."""
    rows, vocab = z.shape
    loss, stats, dz, all_q = np.zeros(rows), np.zeros((rows, 2)), np.zeros((rows, vocab)), np.zeros((rows, vocab))
    for i in range(rows):
        with np.errstate(all="ignore"):
            peak = z[i].max()
            x = np.full(vocab, -np.inf) if peak == -np.inf else (z[i] - peak) / tau
            log_sum = np.log(np.exp(x).sum())
            stats[i] = peak, log_sum
            q = all_q[i] = np.zeros(vocab) if peak == -np.inf else np.exp(x - log_sum)
            there = (ids[i] >= 0) & (ids[i] < vocab) & (t[i] != -np.inf)
            if not there.any():
                continue
            e = np.exp(t[i][there] / tau - (t[i][there] / tau).max())
            p, place = e / e.sum(), ids[i][there]
            if np.isnan(p).any():
                loss[i] = np.nan
            for pn, at in zip(p, place):
                if pn > 0:
                    loss[i] += tau * tau * pn * (np.log(pn) - (-np.inf if peak == -np.inf else x[at] - log_sum))
            if grad is not None and grad[i] != 0:
                teacher = np.zeros(vocab)
                np.add.at(teacher, place, p)
                dz[i] = np.nan if np.isnan(p).any() else tau * grad[i] * (q - teacher)
    return loss, stats, dz, all_q


def small_form(rows, cols, seed):
    """(codes, scales, values) of a random matrix whose products are exact in 32 bits in any order: magnitudes up to 2 and scales of 1
    and 2, so that a product of two elements is a multiple of 1/4 and at most 16, and 2^18 of them stay within 2^24 quarters."""
    assert cols <= 2 ** 18
    rng = np.random.default_rng(seed)
    groups = -(-cols // 128)
    nibbles = rng.integers(0, 5, (rows, groups * 128)) + 8 * rng.integers(0, 2, (rows, groups * 128))
    nibbles[:, cols:] = 0
    scales = rng.integers(127, 129, (groups, rows, 4)).astype(np.uint8)
    scales[np.broadcast_to((np.arange(groups * 4).reshape(groups, 1, 4) * 32 >= cols), scales.shape)] = 0
    codes = (nibbles[:, 0::2] | nibbles[:, 1::2] << 4).astype(np.uint8)
    return codes, scales, mx_values(codes, scales, cols)


# Products over a long axis of matrices made by small_form, and linear layers of tokens made by small_tokens.
LONG_PRODUCTS = [(64, 64, 8192), (70, 130, 8100), (17, 33, 20_001), (300, 500, 16_384), (1, 40, 200_000), (129, 65, 65_665)]
LONG_LINEARS = [(1, 70, 177_280), (1, 70, 177_281), (2, 70, 32_768), (2, 70, 32_769), (5, 70, 8_192), (16, 70, 2_176), (16, 70, 2_177),
                (16, 70, 11_000), (32, 70, 5_000), (33, 70, 20_000)]


def small_tokens(rows, cols, seed):
    """Multiples of 1/2 up to 2, which 4-bit form holds whatever the largest of their block is; the last column is not 0."""
    x = np.random.default_rng(seed).integers(-4, 5, (rows, cols)) / 2.0
    x[:, -1] = 1.5
    return x


def draws_of_all(rows, cols, seed, worker, step, first_row=0, first_col=0):
    """draws(), all elements at a time, of a part of a matrix."""
    assert first_col % 8 == 0
    u = np.uint64
    mask = u(0xFFFFFFFF)
    c0, c1 = np.meshgrid(np.arange(-(-cols // 8), dtype=np.uint64) + u(first_col // 8), np.arange(rows, dtype=np.uint64) + u(first_row))
    c2, c3 = np.full_like(c0, worker), np.full_like(c0, step)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF
    for _ in range(10):
        p0, p1 = c0 * u(0xD2511F53), c2 * u(0xCD9E8D57)
        c0, c1, c2, c3 = p1 >> u(32) ^ c1 ^ u(k0), p1 & mask, p0 >> u(32) ^ c3 ^ u(k1), p0 & mask
        k0, k1 = k0 + 0x9E3779B9 & 0xFFFFFFFF, k1 + 0xBB67AE85 & 0xFFFFFFFF
    low, high = u(0xFFFF), u(16)
    words = np.stack([v for c in (c0, c1, c2, c3) for v in (c & low, c >> high)], axis=2)
    return words.reshape(rows, -1)[:, :cols].astype(np.int64)


def mx_form_of_all(x, r=None):
    """mx_form(), all blocks at a time."""
    rows, cols = x.shape
    groups = -(-cols // 128)
    fill = lambda v: np.pad(v, ((0, 0), (0, groups * 128 - cols))).reshape(rows, groups * 4, 32)
    v, there = fill(x), np.arange(groups * 4) * 32 < cols
    a = np.abs(v)
    whole = np.isfinite(a).all(axis=2)
    largest = np.where(whole, a.max(axis=2), 0.0)
    mantissa, e = np.frexp(largest)
    byte = np.where(largest > 0, np.maximum(e - 3 + ((mantissa > 0.75) if r is not None else 0) + 127, 0), 0)
    t = np.where(whole[:, :, None], a, 0.0) * np.exp2(127.0 - byte)[:, :, None]
    low = np.searchsorted(GRID, np.minimum(t, 6.0), side="right") - 1
    below, above = GRID[low], GRID[np.minimum(low + 1, 7)]
    share = np.where(low < 7, (np.minimum(t, 6.0) - below) / np.where(low < 7, above - below, 1.0), 0.0)
    if r is None:
        up = (share > 0.5) | ((share == 0.5) & (low % 2 == 1))
    else:
        up = np.floor(share * 65536).astype(np.int64) + fill(r) >= 65536
    code = np.where(whole[:, :, None], low + (up & (low < 7)) + 8 * np.signbit(v), 0).astype(np.uint8).reshape(rows, -1)
    code[:, cols:] = 0
    scales = np.where(there, np.where(whole, byte, 255), 0).astype(np.uint8).reshape(rows, groups, 4).transpose(1, 0, 2)
    return code[:, 0::2] | code[:, 1::2] << 4, np.ascontiguousarray(scales)


def hard_matrix(rows, cols, dtype, seed):
    """Heavy-tailed values with both zeros, ties of the grid, subnormal numbers, the largest finite ones, infinities and NaN."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(1.5 * rng.standard_normal((rows, cols))) * 0.03
    pick = lambda share: rng.random((rows, cols)) < share
    x[pick(0.05)] = 0.0
    x[pick(0.02)] = -0.0
    x[::3] = np.where(pick(0.3)[::3], rng.integers(-28, 29, x[::3].shape) / 4.0, x[::3])
    x[1::5] *= 2.0 ** (-12 if dtype == "f16" else -128)
    x[2::7, ::2] = torch.finfo(TYPES[dtype]).max
    x[pick(0.002)] = np.nan
    x[pick(0.002)] = -np.inf
    return torch.from_numpy(x).to(TYPES[dtype])
