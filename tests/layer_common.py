"""Plain 64-bit statements of layer norm, 8-bit integer matrices and Newton-Schulz steps, written from their definitions (tq_norm.h,
tq_i8.h, tq_orth.h), and bounds of the kernels' errors, for their tests."""
import numpy as np
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}        # the smallest magnitude of a type, for subnormal results
U = 2.0 ** -24
QUINTIC = (3.4445, -4.7750, 2.0315)


def strided(t, extra, offset=0, device="cuda"):
    """t on the device as a slice of a wider matrix, `offset` elements into its storage."""
    rows, cols = t.shape
    flat = torch.full((offset + rows * (cols + extra),), float("nan"), dtype=t.dtype, device=device)
    view = flat[offset:].view(rows, cols + extra)[:, :cols]
    view.copy_(t)
    return view


# ---- layer norm

def norm_sums(cols):
    """Additions that a sum over a row goes through: a lane's own, 6 levels of a wavefront, 16 wavefronts."""
    return max(16, -(-cols // 1024) + 8) + 6 + 16


def norm_forward(x, w, b, eps):
    """y, h, mean, 1 / deviation of float64 rows."""
    n = x.shape[1]
    mean = x.sum(dim=1, keepdim=True) / n
    d = x - mean
    r = 1 / torch.sqrt((d * d).sum(dim=1, keepdim=True) / n + eps)
    h = d * r
    y = h if w is None else h * w
    return (y if b is None else y + b), h, mean, r


def norm_forward_bound(y, h, w, b, cols, dtype):
    """The sum of d = x - m (m: a first mean, rounded) is off by k u sum|d|, that of d^2 by k u of itself, so that h is off by
    (k / 2 + 4) u of itself and by k u of the deviation; then a product and a sum, each rounded, and y's own rounding."""
    k = norm_sums(cols)
    ww = torch.ones_like(h) if w is None else w.abs().expand_as(h)
    off = ww * (h.abs() * (k / 2 + 8) + k + 4) * U + 2 * U * y.abs()
    if b is not None:
        off = off + 2 * U * b.abs()
    return HALF_ULP[dtype] * (y.abs() + off) + off + TINY[dtype]


def norm_backward(dy, h, w, r):
    n = dy.shape[1]
    g = dy if w is None else dy * w
    dx = r * (g - g.sum(dim=1, keepdim=True) / n - h * ((g * h).sum(dim=1, keepdim=True) / n))
    return dx, (dy * h).sum(dim=0), dy.sum(dim=0)


def norm_backward_bounds(x, dy, h, w, mean, r, dtype, rows_in_turn):
    """h from statistics that are rounded to binary32: off by u |m| r and by (k / 2 + 8) u of itself, and k u.  The row's two sums: k u of the sums of
    magnitudes and what h's error adds; dweight: a chain of `rows_in_turn` additions."""
    k = norm_sums(dy.shape[1])
    g = dy if w is None else dy * w
    dh = (2 * mean.abs() * r + h.abs() * (k / 2 + 8) + k) * U
    mean_of = lambda t: t.sum(dim=1, keepdim=True) / t.shape[1]
    s1, s2 = mean_of(g.abs()), mean_of((g * h).abs())
    off1 = (k + 4) * U * s1
    off2 = (k + 6) * U * s2 + mean_of(g.abs() * dh)
    exact = norm_backward(dy, h, w, r)
    dx = exact[0]
    off = r * (4 * U * (g.abs() + s1 + h.abs() * s2) + off1 + h.abs() * off2 + dh * (s2 + off2)) + (k / 2 + 8) * U * dx.abs()
    dw = (dy.abs() * dh).sum(dim=0) + (rows_in_turn + 4) * U * (dy * h).abs().sum(dim=0)
    db = (rows_in_turn + 4) * U * dy.abs().sum(dim=0)
    return HALF_ULP[dtype] * (dx.abs() + off) + off + TINY[dtype], dw + TINY["f32"], db + TINY["f32"]


# ---- 8-bit integers

def i8_form(x):
    """(codes int8 [rows, 128 G], scales float32) of a float32 numpy matrix.  In binary64 the products below are exact."""
    rows, cols = x.shape
    codes = np.zeros((rows, -(-cols // 128) * 128), dtype=np.int8)
    a = np.abs(x).max(axis=1)
    with np.errstate(invalid="ignore"):
        scales = np.where(np.isfinite(a), a, np.float32("nan")).astype(np.float32) / np.float32(127)
    for i in range(rows):
        if not np.isfinite(a[i]) or a[i] == 0:
            continue
        big = float(a[i])
        t = np.abs(x[i].astype(np.float64)) * 127
        low = np.floor(t / big)
        twice = 2 * (t - low * big)                         # against big: the middle between two codes
        q = np.where((twice > big) | ((twice == big) & (low % 2 == 1)), low + 1, low)
        codes[i, :cols] = np.where(x[i] < 0, -q, q).astype(np.int8)
    return codes, scales.astype(np.float32)


def i8_product(a, sa, b, sb, bias, dtype):
    """The library's result, bit for bit: an exact sum, three binary32 operations, one rounding to the type."""
    sums = torch.from_numpy(a.astype(np.float64)) @ torch.from_numpy(b.astype(np.float64)).t()      # below 2^53: exact
    out = sums.to(torch.int32).to(torch.float32) * torch.from_numpy(sa).view(-1, 1) * torch.from_numpy(sb)
    if bias is not None:
        out = out + torch.from_numpy(bias)
    return out.to(TYPES[dtype])


# ---- Newton-Schulz steps

def newton_schulz(u, coefficients, eps, rounded=None):
    """The steps in float64; `rounded` is applied to whatever is held between products."""
    rounded = rounded or (lambda t: t)
    flip = u.shape[0] > u.shape[1]
    x = u / (torch.sqrt((u * u).sum()) + eps)
    x = rounded(x.t().contiguous() if flip else x)
    one = torch.eye(x.shape[0], dtype=torch.float64, device=u.device)
    for i, (a, b, c) in enumerate(coefficients):
        gram = rounded(x @ x.t().contiguous())
        x = rounded(a * one + b * gram + c * (gram @ gram)) @ x
        if i + 1 < len(coefficients):
            x = rounded(x)
    return x.t().contiguous() if flip else x


def half(t):
    """As the kernels hold it in binary16."""
    return (t * 4096).to(torch.float16).double() / 4096


def pair(t):
    high = (t * 4096).to(torch.float16)
    return (high.double() + ((t * 4096).float() - high.float()).to(torch.float16).double()) / 4096


def newton_schulz_bound(u, coefficients, eps, unit, sums):
    """How far steps may be from newton_schulz, in the Frobenius norm, when what is held between products has a relative error of `unit` and
    a product's sums of `sums`, relative to the sum of magnitudes.  A step's map X -> p(X) has a derivative whose norm is the largest
    of |p'(s)| and of |p(s) - p(t)| / |s - t|, |p(s) + p(t)| / (s + t) over singular values s, t, all of which the largest |p'| bounds.
    Where an element is subnormal in binary16, times 2^12, it is off by up to 2^-25 * 2^-12 whatever its size."""
    x = (u if u.shape[0] <= u.shape[1] else u.t()) / (torch.sqrt((u * u).sum()) + eps)
    one = torch.eye(x.shape[0], dtype=torch.float64, device=u.device)
    least = 2.0 ** -37 * x.numel() ** 0.5, 2.0 ** -37 * x.shape[0]         # of X, of A and B
    far = unit * float(x.norm()) + least[0]
    for a, b, c in coefficients:
        top = float(torch.linalg.matrix_norm(x, 2)) + far
        s = np.linspace(0, top, 2001)
        slope = np.abs(a + 3 * b * s ** 2 + 5 * c * s ** 4).max()
        gram = x @ x.t().contiguous()
        factor = a * one + b * gram + c * (gram @ gram)
        size, grams, top2 = float(x.norm()), float(gram.norm()), top * top
        off_gram = unit * grams + sums * size * size + least[1]
        off_factor = unit * float(factor.norm()) + least[1] + sums * abs(c) * grams * grams + (abs(b) + 2 * abs(c) * (top2 + off_gram)) * off_gram
        x = factor @ x
        far = slope * far + top * off_factor + unit * float(x.norm()) + least[0] + sums * float(factor.norm()) * size
    return far
