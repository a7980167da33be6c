"""Performance cases of the operators around a student's products: layer norm, 8-bit integer matrices, orthogonalised updates.

A case is a dict of plain values; `op` says which operator it runs:
  "norm"    layer norm of the rows of x: y = (x - mean) / sqrt(var + eps) * weight + bias; with `train` the backward pass too:
            dx and the gradients of weight and bias, which are sums over the rows (rows, cols, dtype, train)
  "cast"    a matrix to 8-bit integers with a scale for each row, and back to the values that they stand for (rows, cols, dtype)
  "product" out = A B^T of two matrices in that form, A [m, k], B [n, k] (out)
  "linear"  out = Q(x) W^T (+ bias): x [m, k] as it comes from the layer before, W [n, k] in that form (dtype, bias)
  "orth"    the orthogonal factor of a matrix by Newton-Schulz steps (rows, cols, dtype)
  "update"  a server's step for `count` matrices: momentum, the orthogonal factor of the result, weight decay, new parameters
            (count, rows, cols, dtype: the gradients' type; parameters and momentum are fp32)

The 8-bit form: with A the largest magnitude of a row, its scale is A / 127 in fp32, an element's code is 127 x / A rounded to the
nearest whole number, ties to even; NaN as the scale of a row that holds a NaN or an infinity.  A row of codes is padded with
zeros to a multiple of 128.
Newton-Schulz: X = U / (|U|_F + EPS), transposed if it has more rows than columns; STEPS times X <- (a I + b A + c A A) X,
A = X X^T, (a, b, c) = QUINTIC, which drives the singular values to about 1; transposed back.
The update: v' = MOMENTUM v + g, U = g + MOMENTUM v', theta' = theta - ETA (scale O + DECAY theta), scale = sqrt(max(1, rows / cols)).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
NORM_EPS = 1e-5
STEPS, EPS = 5, 1e-7
QUINTIC = (3.4445, -4.7750, 2.0315)
ETA, MOMENTUM, DECAY = 0.02, 0.95, 0.01


def _norm(name, rows, cols, dtype, train):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "train": train}


def _cast(name, rows, cols, dtype):
    return {"name": name, "op": "cast", "rows": rows, "cols": cols, "dtype": dtype}


def _product(name, m, n, k, out):
    return {"name": name, "op": "product", "m": m, "n": n, "k": k, "out": out}


def _linear(name, m, n, k, dtype, bias):
    return {"name": name, "op": "linear", "m": m, "n": n, "k": k, "dtype": dtype, "bias": bias}


def _orth(name, rows, cols, dtype):
    return {"name": name, "op": "orth", "rows": rows, "cols": cols, "dtype": dtype}


def _update(name, count, rows, cols, dtype):
    return {"name": name, "op": "update", "count": count, "rows": rows, "cols": cols, "dtype": dtype}


def listed():
    return [
        # One token on its way through a served model: latency.
        _norm("norm-1x4096-bf16", 1, 4096, "bf16", False),
        # A training step's norm, odd sizes, fp32.
        _norm("norm-4099x1001-f32-train", 4099, 1001, "f32", True),
        # A long batch of a wide layer: memory.
        _norm("norm-16384x4096-bf16-train", 16384, 4096, "bf16", True),
        # The activations of a batch with an odd width, fp32.
        _cast("cast-2056x4097-f32", 2056, 4097, "f32"),
        # A large square product in bf16: the matrix rate.
        _product("product-8192-bf16", 8192, 8192, 8192, "bf16"),
        # One token through a large layer: the weights are read once, nothing else counts.
        _linear("linear-1x8192x8192-bf16", 1, 8192, 8192, "bf16", False),
        # A batch of requests, a token each.
        _linear("linear-24x14336x4096-bf16", 24, 14336, 4096, "bf16", True),
        # A prompt with an odd number of tokens through a wide layer.
        _linear("linear-1037x8192x4096-f16", 1037, 8192, 4096, "f16", True),
        # A small matrix: launches.
        _orth("orth-64x256-bf16", 64, 256, "bf16"),
        # A large layer's momentum, as it is sent on in bf16: the matrix rate.
        _orth("orth-4096x4096-bf16", 4096, 4096, "bf16"),
        # The last layer of a small student, fp32 throughout.
        _update("update-1000x784-f32", 1, 1000, 784, "f32"),
        # Four equal layers of a model at once, parameters and momentum in fp32.
        _update("update-4x1024x4096-f32", 4, 1024, 4096, "f32"),
    ]


def _log(rng, low, high):
    """A whole number between low and high, spread over its logarithm; half of the large ones odd, half of them multiples of 160."""
    n = max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))
    if n > 2048:
        n = n - 1 | 1 if rng.random() < 0.5 else n - n % 160
    return n


def draw(rng):
    """One more case of the listed ones' ranges."""
    op = rng.choice(["norm", "cast", "product", "linear", "orth", "update"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op == "norm":
        cols = _log(rng, 1, 32768)
        return _norm(None, _log(rng, 1, min(16384, (1 << 26) // cols)), cols, dtype, rng.random() < 0.7)
    if op == "cast":
        cols = _log(rng, 1, 32768)
        return _cast(None, _log(rng, 1, min(8192, (1 << 26) // cols)), cols, dtype)
    if op == "product":
        return _product(None, _log(rng, 1, 8192), _log(rng, 1, 8192), _log(rng, 1, 8192), dtype)
    if op == "linear":
        return _linear(None, _log(rng, 1, 2048), _log(rng, 64, 8192), _log(rng, 64, 8192), dtype, rng.random() < 0.5)
    if op == "orth":
        return _orth(None, _log(rng, 1, 4096), _log(rng, 1, 4096) if dtype != "f32" else _log(rng, 1, 2048), dtype)
    count, rows = rng.choice([1, 1, 2, 3, 5]), _log(rng, 16, 2048)
    return _update(None, count, rows, _log(rng, 16, 2048 if count > 2 else 4096), dtype)


def _steps_flops(rows, cols):
    """Of the Newton-Schulz steps; X X^T and A A are symmetric, which halves them."""
    r, c = min(rows, cols), max(rows, cols)
    return STEPS * (r * r * c + r ** 3 + 2 * r * r * c)


def work(case):
    """Each input read and each output written once by every call; a product's multiplications and additions."""
    op = case["op"]
    if op == "norm":
        n, size = case["rows"] * case["cols"], SIZE[case["dtype"]]
        return {"bytes": n * size * (5 if case["train"] else 2) + 8 * case["cols"] * (3 if case["train"] else 1), "flops": n * (22 if case["train"] else 8)}
    if op == "cast":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (SIZE[case["dtype"]] + 1 + 1 + 4), "flops": 4 * n}
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * (k + 4) + m * n * SIZE[case["out"]], "flops": 2 * m * n * k}
    if op == "linear":
        m, n, k, size = case["m"], case["n"], case["k"], SIZE[case["dtype"]]
        return {"bytes": n * (k + 4 + 4 * case["bias"]) + (m * k + m * n) * size, "flops": 2 * m * n * k}
    n = case["rows"] * case["cols"]
    if op == "orth":
        return {"bytes": 2 * n * SIZE[case["dtype"]], "flops": _steps_flops(case["rows"], case["cols"])}
    return {"bytes": case["count"] * n * (16 + SIZE[case["dtype"]]), "flops": case["count"] * _steps_flops(case["rows"], case["cols"])}


# ---- inputs

def _generator(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 1000 + salt)


def _normal(seed, salt, shape, scale=1.0):
    return torch.randn(shape, generator=_generator(seed, salt), device="cuda") * scale


def _activations(seed, salt, shape):
    """Rows of different size, each about a mean of its own, a few channels far larger than the others."""
    rows, cols = shape
    x = _normal(seed, salt, shape) * torch.exp(0.5 * _normal(seed, salt + 1, (rows, 1))) + 0.5 * _normal(seed, salt + 2, (rows, 1))
    x[:, seed % 11::97] *= 8
    return x


def _gradient(seed, salt, shape, scale):
    """Magnitudes spread over several octaves from one element to the next, a few directions above the others, a few rows without
    any (ids that did not occur)."""
    x = _normal(seed, salt, shape) * torch.exp(0.8 * _normal(seed, salt + 1, shape))
    few = min(4, *shape)
    x += 0.5 * _normal(seed, salt + 2, (shape[0], few)) @ _normal(seed, salt + 3, (few, shape[1]))
    if shape[0] > 64:
        x[seed % 7::61] = 0
    return x * scale


def _random_form(seed, salt, rows, cols):
    """A weight or activation matrix in the 8-bit form."""
    padded = -(-cols // 128) * 128
    codes = torch.round(_normal(seed, salt, (rows, padded), 36.0)).clamp_(-127, 127).to(torch.int8)
    codes[:, cols:] = 0
    scales = torch.exp(0.3 * _normal(seed, salt + 1, (rows,))) * (0.02 / cols ** 0.5)
    return codes, scales


def prepare(case, seed):
    op = case["op"]
    s = {"case": case}
    if op == "norm":
        shape, dtype = (case["rows"], case["cols"]), TYPES[case["dtype"]]
        s["x"] = _activations(seed, 1, shape).to(dtype)
        s["weight"] = 1 + 0.2 * _normal(seed, 5, (case["cols"],))
        s["bias"] = 0.1 * _normal(seed, 6, (case["cols"],))
        if case["train"]:
            s["dy"] = _normal(seed, 7, shape, 1e-2).to(dtype)
    elif op == "cast":
        s["x"] = _activations(seed, 1, (case["rows"], case["cols"])).to(TYPES[case["dtype"]])
    elif op == "product":
        s["a"] = _random_form(seed, 1, case["m"], case["k"])
        s["b"] = _random_form(seed, 3, case["n"], case["k"])
    elif op == "linear":
        s["x"] = _activations(seed, 1, (case["m"], case["k"])).to(TYPES[case["dtype"]])
        s["w"] = _random_form(seed, 4, case["n"], case["k"])
        s["bias"] = _normal(seed, 6, (case["n"],), 0.1) if case["bias"] else None
    elif op == "orth":
        s["g"] = _gradient(seed, 1, (case["rows"], case["cols"]), 1e-3).to(TYPES[case["dtype"]])
    else:
        shape, many = (case["rows"], case["cols"]), range(case["count"])
        s["gs"] = [_gradient(seed, 10 * i + 1, shape, 1e-3).to(TYPES[case["dtype"]]) for i in many]
        s["velocities"] = [_gradient(seed, 10 * i + 5, shape, 1e-2) for i in many]
        s["thetas"] = [_normal(seed, 10 * i + 9, shape, case["cols"] ** -0.5) for i in many]
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The buffers that a program keeps from step to step."""
    from paper_2402_01798_amd import binding as tq
    case = s["case"]
    op = case["op"]
    dev = "cuda"

    def workspace(nbytes):
        return torch.empty(nbytes, dtype=torch.uint8, device=dev)

    if op == "norm":
        s["y"] = torch.empty_like(s["x"])
        s["stats"] = torch.empty(case["rows"], 2, device=dev)
        if case["train"]:
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
            s["ws"] = workspace(tq.layernorm_workspace_bytes(case["rows"], case["cols"]))
    elif op == "cast":
        s["form"] = tq.alloc_i8(case["rows"], case["cols"])
        s["values"] = torch.empty(case["rows"], case["cols"], device=dev)
    elif op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"], s["b"] = tq.I8Matrix(*s["a"], m, k), tq.I8Matrix(*s["b"], n, k)
        s["out"] = torch.empty(m, n, dtype=TYPES[case["out"]], device=dev)
        s["ws"] = workspace(tq.i8_matmul_workspace_bytes(m, n, k))
    elif op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s["w"] = tq.I8Matrix(*s["w"], n, k)
        s["out"] = torch.empty(m, n, dtype=TYPES[case["dtype"]], device=dev)
        s["ws"] = workspace(tq.i8_linear_workspace_bytes(m, n, k))
    elif op == "orth":
        s["out"] = torch.empty_like(s["g"])
        s["ws"] = workspace(tq.orthogonalize_workspace_bytes(case["rows"], case["cols"], 1, tq.ORTH_SPLIT))
    else:
        s["new_velocities"] = [torch.empty_like(v) for v in s["velocities"]]
        s["new_thetas"] = [torch.empty_like(t) for t in s["thetas"]]
        s["ws"] = workspace(tq.orthogonalize_workspace_bytes(case["rows"], case["cols"], case["count"], tq.ORTH_SPLIT))


def _scale(case):
    return max(1.0, case["rows"] / case["cols"]) ** 0.5


# ---- one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2402_01798_amd import binding as tq
    case = s["case"]
    op = case["op"]
    if op == "norm":
        tq.tq_layernorm_forward(s["x"], s["weight"], s["bias"], s["y"], s["stats"], eps=NORM_EPS)
        if not case["train"]:
            return s["y"]
        tq.tq_layernorm_backward(s["x"], s["dy"], s["weight"], s["stats"], s["dx"], s["dweight"], s["dbias"], s["ws"])
        return [s["y"], s["dx"], s["dweight"], s["dbias"]]
    if op == "cast":
        tq.tq_i8_quantize(s["x"], s["form"])
        return tq.tq_i8_dequantize(s["form"], s["values"])
    if op == "product":
        return tq.tq_i8_matmul(s["a"], s["b"], s["out"], s["ws"])
    if op == "linear":
        return tq.tq_i8_linear(s["x"], s["w"], s["out"], s["ws"], bias=s["bias"])
    if op == "orth":
        return tq.tq_orthogonalize(s["g"], s["out"], s["ws"], steps=STEPS, precision=tq.ORTH_SPLIT, eps=EPS)
    tq.tq_orthogonal_update_multi(s["gs"], s["velocities"], s["thetas"], s["ws"], eta=ETA, momentum=MOMENTUM, nesterov=True,
                                  weight_decay=DECAY, scale=_scale(case), steps=STEPS, precision=tq.ORTH_SPLIT, eps=EPS,
                                  velocities_out=s["new_velocities"], thetas_out=s["new_thetas"])
    return [s["new_velocities"], s["new_thetas"]]


def _plain_norm(case, s):
    x, weight, dtype = s["x"].float(), s["weight"], s["x"].dtype
    mean = x.mean(dim=1, keepdim=True)
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).mean(dim=1, keepdim=True) + NORM_EPS)
    h = d * rstd
    y = (h * weight + s["bias"]).to(dtype)
    if not case["train"]:
        return y
    dy = s["dy"].float()
    g = dy * weight
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - h * (g * h).mean(dim=1, keepdim=True))
    return [y, dx.to(dtype), (dy * h).sum(dim=0), dy.sum(dim=0)]


def _plain_cast(x):
    """Codes (fp32 numbers) and scales.  The quotient in 64 bits: in 32 its own rounding takes it past a border now and then."""
    largest = x.float().abs().amax(dim=1, keepdim=True)
    fine = torch.isfinite(largest)
    codes = torch.round(x.double() * 127 / largest.double()).float()
    codes = torch.where(fine & (largest > 0), codes, 0.0)
    return codes, torch.where(fine, largest / 127, math.nan)


def _plain_steps(u):
    flip = u.shape[0] > u.shape[1]
    x = u / (torch.sqrt((u.double() * u.double()).sum()) + EPS).float()
    if flip:
        x = x.t().contiguous()
    a, b, c = QUINTIC
    for _ in range(STEPS):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if flip else x


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "norm":
        return _plain_norm(case, s)
    if op == "cast":
        codes, scales = _plain_cast(s["x"])
        return codes * scales
    if op == "product":
        (a, sa), (b, sb) = s["a"], s["b"]
        return ((a.float() @ b.float().t()) * sa.view(-1, 1) * sb).to(TYPES[case["out"]])
    if op == "linear":
        codes, scales = _plain_cast(s["x"])
        w, sw = s["w"]
        out = (codes @ w[:, :case["k"]].float().t()) * scales * sw
        return (out if s["bias"] is None else out + s["bias"]).to(s["x"].dtype)
    if op == "orth":
        return _plain_steps(s["g"].float()).to(s["g"].dtype).contiguous()
    velocities, thetas = [], []
    for g, v, theta in zip(s["gs"], s["velocities"], s["thetas"]):
        g = g.float()
        v = MOMENTUM * v + g
        velocities.append(v)
        thetas.append(theta - ETA * (_scale(case) * _plain_steps(g + MOMENTUM * v) + DECAY * theta))
    return [velocities, thetas]


# ---- the definition in 64 bits

def _exact_codes(x):
    """Every element to the whole number that lies nearest, by its distances to the two beside it; ties to the even one."""
    largest = x.abs().amax(dim=1, keepdim=True)
    usable = torch.isfinite(largest) & (largest > 0)
    unit = torch.where(usable, largest, 1.0)
    t = torch.where(usable, x, 0.0).abs() * 127
    low = torch.floor(t / unit)
    below, above = t - low * unit, (low + 1) * unit - t
    q = torch.where((above < below) | ((above == below) & (low % 2 == 1)), low + 1, low)
    return torch.copysign(q, x), torch.where(torch.isfinite(largest), largest / 127, math.nan)


def _exact_orthogonal(u):
    x = u / (torch.linalg.vector_norm(u) + EPS)
    wide = x if x.shape[0] <= x.shape[1] else x.t().contiguous()
    a, b, c = QUINTIC
    one = torch.eye(wide.shape[0], dtype=torch.float64, device=wide.device)
    for _ in range(STEPS):
        gram = wide @ wide.t().contiguous()
        wide = (a * one + gram @ (b * one + c * gram)) @ wide
    return wide if x.shape[0] <= x.shape[1] else wide.t()


def exact(case, seed):
    global own
    held, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = held
    op = case["op"]
    if op == "norm":
        x, weight, bias = s["x"].double(), s["weight"].double(), s["bias"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        deviation = torch.sqrt(var + NORM_EPS)
        h = (x - mean) / deviation
        y = h * weight + bias
        if not case["train"]:
            return y
        dy = s["dy"].double()
        g = dy * weight
        dx = (g - (g.sum(dim=1, keepdim=True) + h * (g * h).sum(dim=1, keepdim=True)) / case["cols"]) / deviation
        return [y, dx, torch.linalg.vecdot(dy, h, dim=0), dy.sum(dim=0)]
    if op == "cast":
        codes, scales = _exact_codes(s["x"].double())
        return codes * scales
    if op == "product":
        (a, sa), (b, sb) = s["a"], s["b"]
        return (a.double() * sa.double().view(-1, 1)) @ (b.double() * sb.double().view(-1, 1)).t().contiguous()
    if op == "linear":
        codes, scales = _exact_codes(s["x"].double())
        w, sw = s["w"]
        out = (codes * scales) @ (w[:, :case["k"]].double() * sw.double().view(-1, 1)).t().contiguous()
        return out if s["bias"] is None else out + s["bias"].double()
    if op == "orth":
        return _exact_orthogonal(s["g"].double()).contiguous()
    velocities, thetas = [], []
    for g, v, theta in zip(s["gs"], s["velocities"], s["thetas"]):
        v = MOMENTUM * v.double() + g.double()
        velocities.append(v)
        thetas.append(theta.double() * (1 - ETA * DECAY) - ETA * _scale(case) * _exact_orthogonal(g.double() + MOMENTUM * v))
    return [velocities, thetas]
