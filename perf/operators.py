"""Performance cases of the operators that make and use a student's gradients: microscaled 4-bit matrices and distillation.

A case is a dict of plain values; `op` says which operator it runs:
  "cast"     a matrix to microscaled 4-bit form and back to the values it stands for: as it is, transposed, or both
             (rows, cols, dtype, form "rows" / "cols" / "both", stochastic)
  "product"  out = A B^T (+ add) of two matrices in that form, A [m, k], B [n, k] (out, add)
  "linear"   out = x W^T, x [m, k] as it comes from the layer before, W [n, k] in that form (dtype)
  "train"    a linear layer's training step in that form: y = x W^T, dx = dy W, dW = dy^T x, x and W rounded to nearest, dy
             stochastically, everything cast anew because every step brings another x, W and dy (tokens, inputs, outputs, dtype)
  "distill"  the loss against a teacher's top logits and its gradient (rows, vocab, top, dtype, temperature): `fused` in one
             call, for a program that knows the rows' weights beforehand, else the loss first and the gradient later

The 4-bit form (OCP microscaling, MXFP4): 32 consecutive elements of a row share a scale 2^(s - 127), s one byte, 255 for a
block that holds a NaN or an infinity; an element is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  With A the block's largest
magnitude, nearest rounding (ties to even, beyond 6 to 6) takes the scale 2^(floor(log2 A) - 2), stochastic rounding the
smallest power of two with A <= 6 * scale, so that nothing is clipped and the mean of the draws is the value.  Element
(i, j)'s draw is the 16 bits at place j % 8 of Philox4x32-10 with the counter (j / 8, i, worker, step) and the key `seed`,
also where the transposed matrix is written.
Codes: row-major, two in a byte, the even element low, a row padded with zeros to a multiple of 128 elements; scales:
[groups of 128 elements, rows, 4], 0 where there is no element.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
WORKER, STEP = 3, 11


def _cast(name, rows, cols, dtype, form, stochastic):
    return {"name": name, "op": "cast", "rows": rows, "cols": cols, "dtype": dtype, "form": form, "stochastic": stochastic}


def _product(name, m, n, k, out, add):
    return {"name": name, "op": "product", "m": m, "n": n, "k": k, "out": out, "add": add}


def _linear(name, m, n, k, dtype):
    return {"name": name, "op": "linear", "m": m, "n": n, "k": k, "dtype": dtype}


def _train(name, tokens, inputs, outputs, dtype):
    return {"name": name, "op": "train", "tokens": tokens, "inputs": inputs, "outputs": outputs, "dtype": dtype}


def _distill(name, rows, vocab, top, dtype, temperature, fused):
    return {"name": name, "op": "distill", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "temperature": temperature,
            "fused": fused}


def listed():
    return [
        # The activations of a few tokens with an odd width, fp32: latency.
        _cast("cast-61x1001-f32", 61, 1001, "f32", "rows", False),
        # A large layer's output gradient, both ways, as the two products of a backward pass want it.
        _cast("cast-8192x8192-bf16-both", 8192, 8192, "bf16", "both", True),
        # A weight gradient of a batch with an odd number of tokens, added to what earlier batches left, in fp32.
        _product("product-2056x1000x1999-f32-add", 2056, 1000, 1999, "f32", True),
        # A large square product in bf16: the matrix rate.
        _product("product-8192-bf16", 8192, 8192, 8192, "bf16", False),
        # One token through a large layer: the weights are read once, nothing else counts.
        _linear("linear-1x8192x8192", 1, 8192, 8192, "bf16"),
        # A prompt with an odd number of tokens through a wide layer.
        _linear("linear-1037x8192x4096-f16", 1037, 8192, 4096, "f16"),
        # A small layer's training step on a short batch, fp32 throughout: latency and launches.
        _train("train-64x784x1000-f32", 64, 784, 1000, "f32"),
        # A large layer's training step on a long batch.
        _train("train-4096x4096x8192-bf16", 4096, 4096, 8192, "bf16"),
        # A few rows of a large odd-sized vocabulary in fp32, the loss first and the gradient when the program asks for it.
        _distill("distill-7x50001-f32-apart", 7, 50001, 20, "f32", 1.0, False),
        # A batch of rows, the loss and the gradient apart.
        _distill("distill-4096x32000-bf16-apart", 4096, 32000, 64, "bf16", 2.0, False),
        # One row of a small vocabulary: latency.
        _distill("distill-1x8192-bf16", 1, 8192, 8, "bf16", 1.0, True),
        # A batch of rows of a large odd-sized vocabulary, loss and gradient at once.
        _distill("distill-2048x131001-bf16", 2048, 131001, 128, "bf16", 4.0, True),
    ]


def _log(rng, low, high):
    """A whole number between low and high, spread over its logarithm; half of the large ones odd, half of them five blocks
    of 32 times something."""
    n = max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))
    if n > 2048:
        n = n - 1 | 1 if rng.random() < 0.5 else n - n % 160
    return n


def draw(rng):
    """One more case of the listed ones' ranges."""
    op = rng.choice(["cast", "product", "linear", "train", "distill"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op == "cast":
        rows, cols = _log(rng, 1, 8192), _log(rng, 1, 8192)
        return _cast(None, rows, cols, dtype, rng.choice(["rows", "cols", "both"]), rng.random() < 0.5)
    if op == "product":
        return _product(None, _log(rng, 1, 8192), _log(rng, 1, 8192), _log(rng, 1, 8192), dtype, rng.random() < 0.5)
    if op == "linear":
        return _linear(None, _log(rng, 1, 1024), _log(rng, 64, 8192), _log(rng, 64, 4096), dtype)
    if op == "train":
        return _train(None, _log(rng, 1, 4096), _log(rng, 32, 4096), _log(rng, 32, 8192), dtype)
    vocab, fused = _log(rng, 64, 131001), rng.random() < 0.5
    rows = _log(rng, 1, min(4096, 10 ** 9 // (vocab * SIZE[dtype] * (2 if fused else 3))))
    return _distill(None, rows, vocab, _log(rng, 1, min(vocab // 4, 256)), dtype, rng.choice([1.0, 2.0, 4.0]), fused)


def work(case):
    """Each input read and each output written once; a product's multiplications and additions, an exponential counted as one."""
    op = case["op"]
    if op == "cast":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (SIZE[case["dtype"]] + 2 * (2 if case["form"] == "both" else 1)), "flops": 4 * n}
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * _form_bytes(k) + m * n * (SIZE[case["out"]] + 4 * case["add"]), "flops": 2 * m * n * k}
    if op == "linear":
        m, n, k, size = case["m"], case["n"], case["k"], SIZE[case["dtype"]]
        return {"bytes": n * _form_bytes(k) + (m * k + m * n) * size, "flops": 2 * m * n * k}
    if op == "train":
        t, i, o, size = case["tokens"], case["inputs"], case["outputs"], SIZE[case["dtype"]]
        return {"bytes": 2 * (t * i + t * o) * size + i * o * (size + 4), "flops": 6 * t * i * o}
    n = case["rows"] * case["vocab"]
    passes = 2 if case["fused"] else 3
    return {"bytes": n * SIZE[case["dtype"]] * passes + case["rows"] * (case["top"] * 8 + 12), "flops": 6 * n}


def _form_bytes(k):
    return -(-k // 2) + -(-k // 32)


# ---- inputs

def _generator(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 1000 + salt)


def _normal(seed, salt, shape, scale=1.0):
    return torch.randn(shape, generator=_generator(seed, salt), device="cuda") * scale


def _heavy(seed, salt, shape, scale):
    """Gradients: magnitudes spread over several octaves from one element to the next, a few rows without any (masked tokens)."""
    x = _normal(seed, salt, shape, scale) * torch.exp(0.8 * _normal(seed, salt + 1, shape))
    if shape[0] > 8:
        x[seed % 7::61] = 0
    return x


def _random_form(seed, salt, rows, cols):
    """A weight or activation matrix in the 4-bit form: every code, scales within a few octaves."""
    stride, groups = -(-cols // 128) * 64, -(-cols // 128)
    g = _generator(seed, salt)
    codes = torch.randint(0, 256, (rows, stride), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(118, 124, (groups, rows, 4), generator=g, device="cuda", dtype=torch.uint8)
    element = torch.arange(2 * stride, device="cuda").view(-1, 2) < cols
    codes &= element[:, 0].to(torch.uint8) * 15 + element[:, 1].to(torch.uint8) * 240
    block = torch.arange(4 * groups, device="cuda").view(groups, 1, 4) * 32 < cols
    scales *= block.to(torch.uint8)
    return codes, scales


def prepare(case, seed):
    op = case["op"]
    s = {"case": case, "seed": seed}
    if op == "cast":
        s["x"] = _heavy(seed, 1, (case["rows"], case["cols"]), 1e-3 if case["dtype"] != "f16" else 0.1).to(TYPES[case["dtype"]])
    elif op == "product":
        s["a"] = _random_form(seed, 1, case["m"], case["k"])
        s["b"] = _random_form(seed, 2, case["n"], case["k"])
        s["add"] = _normal(seed, 3, (case["m"], case["n"])) if case["add"] else None
    elif op == "linear":
        s["x"] = _normal(seed, 1, (case["m"], case["k"])).to(TYPES[case["dtype"]])
        s["w"] = _random_form(seed, 2, case["n"], case["k"])
    elif op == "train":
        t, i, o, dtype = case["tokens"], case["inputs"], case["outputs"], TYPES[case["dtype"]]
        s["x"] = _normal(seed, 1, (t, i)).to(dtype)
        s["w"] = _normal(seed, 2, (o, i), i ** -0.5).to(dtype)
        s["dy"] = _heavy(seed, 3, (t, o), 1e-2).to(dtype)
    else:
        rows, vocab, top = case["rows"], case["vocab"], case["top"]
        g = _generator(seed, 5)
        z = _normal(seed, 1, (rows, vocab), 3.0)
        pad = vocab // 100
        if pad:
            z[:, vocab - pad:] = -math.inf                  # the vocabulary's padding
        s["z"] = z.to(TYPES[case["dtype"]])
        place = torch.randint(0, vocab, (rows, 1), generator=g, device="cuda", dtype=torch.int32)
        ids = (place + torch.arange(top, device="cuda", dtype=torch.int32) * ((vocab - pad) // top)) % (vocab - pad)
        s["t"] = torch.sort(_normal(seed, 2, (rows, top), 3.0), dim=1, descending=True)[0]
        kept = torch.randint(1, 2 * top + 1, (rows, 1), generator=g, device="cuda")      # a nucleus: half of the rows have fewer
        s["ids"] = ids.masked_fill(torch.arange(top, device="cuda") >= kept, -1).to(torch.int32)
        s["grad"] = torch.rand((rows,), generator=g, device="cuda") / rows
        if rows > 8:
            s["ids"][seed % 5::37] = -1                     # rows without a teacher
            s["grad"][seed % 3::29] = 0                     # rows that do not count
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

    if op == "cast":
        rows, cols = case["rows"], case["cols"]
        if case["form"] != "cols":
            s["form"], s["values"] = tq.alloc_mx(rows, cols), torch.empty(rows, cols, dtype=torch.bfloat16, device=dev)
        if case["form"] != "rows":
            s["form_t"], s["values_t"] = tq.alloc_mx(cols, rows), torch.empty(cols, rows, dtype=torch.bfloat16, device=dev)
    elif op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"], s["b"] = tq.MxMatrix(*s["a"], m, k), tq.MxMatrix(*s["b"], n, k)
        s["out"] = torch.empty(m, n, dtype=TYPES[case["out"]], device=dev)
        s["ws"] = workspace(tq.mx_matmul_workspace_bytes(m, n, k))
    elif op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s["w"] = tq.MxMatrix(*s["w"], n, k)
        s["out"] = torch.empty(m, n, dtype=TYPES[case["dtype"]], device=dev)
        s["ws"] = workspace(tq.mx_linear_workspace_bytes(m, n, k))
    elif op == "train":
        t, i, o, dtype = case["tokens"], case["inputs"], case["outputs"], TYPES[case["dtype"]]
        s["forms"] = [tq.alloc_mx(t, i), tq.alloc_mx(i, t), tq.alloc_mx(o, i), tq.alloc_mx(i, o), tq.alloc_mx(t, o), tq.alloc_mx(o, t)]
        s["y"] = torch.empty(t, o, dtype=dtype, device=dev)
        s["dx"] = torch.empty(t, i, dtype=dtype, device=dev)
        s["dw"] = torch.empty(o, i, dtype=torch.float32, device=dev)
        s["ws"] = workspace(max(tq.mx_matmul_workspace_bytes(*mnk) for mnk in ((t, o, i), (t, i, o), (o, i, t))))
    else:
        rows, vocab = case["rows"], case["vocab"]
        s["loss"] = torch.empty(rows, dtype=torch.float32, device=dev)
        s["stats"] = torch.empty(rows, 2, dtype=torch.float32, device=dev)
        s["dz"] = torch.empty(rows, vocab, dtype=TYPES[case["dtype"]], device=dev)


# ---- one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2402_01798_amd import binding as tq
    case = s["case"]
    op = case["op"]
    if op == "cast":
        form, form_t = s.get("form"), s.get("form_t")
        tq.tq_mx_quantize(s["x"], form, form_t, tq.MX_STOCHASTIC if case["stochastic"] else tq.MX_NEAREST, s["seed"], WORKER, STEP)
        return [tq.tq_mx_dequantize(f, v) for f, v in ((form, s.get("values")), (form_t, s.get("values_t"))) if f is not None]
    if op == "product":
        return tq.tq_mx_matmul(s["a"], s["b"], s["out"], s["ws"], add=s["add"])
    if op == "linear":
        return tq.tq_mx_linear(s["x"], s["w"], s["out"], s["ws"])
    if op == "train":
        x, xt, w, wt, dy, dyt = s["forms"]
        tq.tq_mx_quantize(s["x"], x, xt)
        tq.tq_mx_quantize(s["w"], w, wt)
        tq.tq_mx_quantize(s["dy"], dy, dyt, tq.MX_STOCHASTIC, s["seed"], WORKER, STEP)
        return [tq.tq_mx_matmul(x, w, s["y"], s["ws"]), tq.tq_mx_matmul(dy, wt, s["dx"], s["ws"]),
                tq.tq_mx_matmul(dyt, xt, s["dw"], s["ws"])]
    if case["fused"]:
        tq.tq_distill(s["z"], s["ids"], s["t"], s["grad"], s["loss"], s["dz"], case["temperature"])
        return [s["loss"], s["dz"]]
    tq.tq_distill_forward(s["z"], s["ids"], s["t"], s["loss"], s["stats"], case["temperature"])
    tq.tq_distill_backward(s["z"], s["ids"], s["t"], s["stats"], s["grad"], s["dz"], case["temperature"])
    return [s["loss"], s["dz"]]


def _power(byte):
    """2^(byte - 127) in fp32, NaN for 255."""
    b = byte.to(torch.int32)
    return torch.where(b == 255, 0x7FC00000, torch.where(b == 0, 0x00400000, b << 23)).view(torch.float32)


def _draws(rows, cols, seed):
    """16 bits for each element [rows, cols]."""
    mask = 0xFFFFFFFF
    c0 = torch.arange(-(-cols // 8), device="cuda", dtype=torch.int64).expand(rows, -1)
    c1 = torch.arange(rows, device="cuda", dtype=torch.int64).view(-1, 1).expand_as(c0)
    c2, c3 = torch.full_like(c0, WORKER), torch.full_like(c0, STEP)
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & mask) ^ c1 ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c3 ^ k1, p0 & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    words = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], dim=2)
    return words.reshape(rows, -1)[:, :cols].to(torch.int32)


def _plain_values(x, draws=None):
    """What the 4-bit form of x [rows, cols] stands for, blocks along the rows, in fp32."""
    rows, cols = x.shape
    pad = -cols % 32
    v = torch.nn.functional.pad(x.float(), (0, pad)).view(rows, -1, 32)
    bits = v.abs().amax(dim=2, keepdim=True).view(torch.int32)
    finite = torch.isfinite(v).all(dim=2, keepdim=True)
    exponent = (bits >> 23) - 2
    if draws is not None:
        exponent = exponent + ((bits & 0x7FFFFF) > 0x400000).to(torch.int32)
    byte = exponent.clamp(min=0)
    scaled = v * _power(254 - byte)                         # times 2^(127 - byte)
    a = scaled.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = a / step
    if draws is None:
        q = torch.round(q)
    else:
        low = torch.floor(q)
        up = ((q - low) * 65536).to(torch.int32) + torch.nn.functional.pad(draws, (0, pad)).view_as(v) >= 65536
        q = low + up
    value = torch.copysign((q * step).clamp(max=6.0), v) * _power(byte)
    return torch.where(finite, value, math.nan).view(rows, -1)[:, :cols]


def _form_values(codes, scales, cols):
    """The values of a matrix that is held in the 4-bit form, in fp32."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    rows = codes.shape[0]
    v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], dim=2).view(rows, -1, 32)
    return (v * _power(scales.permute(1, 0, 2).reshape(rows, -1, 1))).view(rows, -1)[:, :cols]


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "cast":
        draws = _draws(case["rows"], case["cols"], s["seed"]) if case["stochastic"] else None
        out = []
        if case["form"] != "cols":
            out.append(_plain_values(s["x"], draws).to(torch.bfloat16))
        if case["form"] != "rows":
            out.append(_plain_values(s["x"].t().contiguous(), None if draws is None else draws.t()).to(torch.bfloat16))
        return out
    if op == "product":
        out = _form_values(*s["a"], case["k"]) @ _form_values(*s["b"], case["k"]).t()
        if s["add"] is not None:
            out += s["add"]
        return out.to(TYPES[case["out"]])
    if op == "linear":
        return (_plain_values(s["x"]) @ _form_values(*s["w"], case["k"]).t()).to(TYPES[case["dtype"]])
    if op == "train":
        dtype = TYPES[case["dtype"]]
        x, w, dy = s["x"], s["w"], s["dy"]
        draws = _draws(case["tokens"], case["outputs"], s["seed"])
        y = _plain_values(x) @ _plain_values(w).t()
        dx = _plain_values(dy, draws) @ _plain_values(w.t().contiguous()).t()
        dw = _plain_values(dy.t().contiguous(), draws.t()) @ _plain_values(x.t().contiguous()).t()
        return [y.to(dtype), dx.to(dtype), dw]
    return _plain_distill(case, s)


def _plain_distill(case, s):
    tau, vocab = case["temperature"], case["vocab"]
    z, ids = s["z"].float() / tau, s["ids"].long()
    present = (ids >= 0) & (ids < vocab) & (s["t"] > -math.inf)
    t = torch.where(present, s["t"] / tau, -math.inf)
    top = t.amax(dim=1, keepdim=True)
    e = torch.where(present, torch.exp(t - top), 0.0)
    total = e.sum(dim=1, keepdim=True)
    p = torch.where(present, e / total, 0.0)
    log_p = t - top - torch.log(total)
    peak = z.amax(dim=1, keepdim=True)
    lse = peak + torch.log(torch.exp(z - peak).sum(dim=1, keepdim=True))
    ids = torch.where(present, ids, 0)
    loss = torch.where(p > 0, p * (log_p - (z.gather(1, ids) - lse)), 0.0).sum(dim=1) * (tau * tau)
    dz = torch.exp(z - lse).scatter_add_(1, ids, -p)
    counts = present.any(dim=1, keepdim=True) & (s["grad"].view(-1, 1) != 0)
    dz = torch.where(counts, dz * (tau * s["grad"].view(-1, 1)), 0.0).to(s["z"].dtype)
    return [loss, dz]


# ---- the definition in 64 bits

def _exact_draws(rows, cols, seed):
    groups = -(-cols // 8)
    u32 = np.uint64(0xFFFFFFFF)
    j, i = np.meshgrid(np.arange(groups, dtype=np.uint64), np.arange(rows, dtype=np.uint64))
    word = [j, i, np.full_like(j, WORKER), np.full_like(j, STEP)]
    key = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]
    for _ in range(10):
        a, b = word[0] * np.uint64(0xD2511F53), word[2] * np.uint64(0xCD9E8D57)
        word = [(b >> np.uint64(32)) ^ word[1] ^ np.uint64(key[0]), b & u32, (a >> np.uint64(32)) ^ word[3] ^ np.uint64(key[1]), a & u32]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    flat = np.empty((rows, groups, 4), dtype=np.uint32)
    for w in range(4):
        flat[:, :, w] = word[w]
    return torch.from_numpy(flat.view(np.uint16).reshape(rows, -1)[:, :cols].astype(np.float64)).cuda()


def _exact_power(byte):
    """2^(byte - 127) in fp64, from a table (a device's exp2 may be off by a unit in the last place)."""
    return torch.tensor([2.0 ** (b - 127) for b in range(255)] + [math.nan], dtype=torch.float64, device="cuda")[byte.long()]


def _exact_block(v, draws):
    """One block of columns [rows, <= 32] in fp64: each element to the magnitude that the definition names."""
    grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    largest = v.abs().amax(dim=1, keepdim=True)
    mantissa, exponent = torch.frexp(largest)               # largest = mantissa * 2^exponent, mantissa in [0.5, 1)
    exponent = exponent - 3
    if draws is not None:
        exponent = exponent + (mantissa > 0.75)
    scale = _exact_power(torch.where(largest > 0, exponent + 127, 0).clamp(0, 254))
    a = v.abs() / scale
    value = torch.zeros_like(a)
    for n in range(7):
        low, high = grid[n], grid[n + 1]
        if draws is None:
            middle = (low + high) / 2
            value = torch.where(a >= middle if n % 2 else a > middle, high, value)
        else:
            share = torch.floor((a - low) / (high - low) * 65536)
            inside = (a >= low) & (a < high)
            value = torch.where(inside, torch.where(share + draws >= 65536, high, low), value)
            value = torch.where(a == high, high, value)
    value = torch.copysign(value * scale, v)
    return torch.where(torch.isfinite(largest), value, math.nan)


def _exact_values(x, draws=None):
    x = x.double()
    cols = range(0, x.shape[1], 32)
    return torch.cat([_exact_block(x[:, c:c + 32], None if draws is None else draws[:, c:c + 32]) for c in cols], dim=1)


def _exact_form(codes, scales, cols):
    nibble = torch.stack([codes % 16, codes // 16], dim=2).view(codes.shape[0], -1)[:, :cols].double()
    magnitude, negative = nibble % 8, nibble >= 8
    value = torch.where(magnitude < 4, magnitude / 2, torch.where(magnitude < 6, magnitude - 2, 2 * magnitude - 8))
    block = _exact_power(scales.permute(1, 0, 2).reshape(codes.shape[0], -1)).repeat_interleave(32, dim=1)[:, :cols]
    return torch.where(negative, -value, value) * block


def exact(case, seed):
    global own
    held, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = held
    op = case["op"]
    if op == "cast":
        draws = _exact_draws(case["rows"], case["cols"], seed) if case["stochastic"] else None
        out = []
        if case["form"] != "cols":
            out.append(_exact_values(s["x"], draws))
        if case["form"] != "rows":
            out.append(_exact_values(s["x"].t(), None if draws is None else draws.t()))
        return out
    if op == "product":
        out = _exact_form(*s["a"], case["k"]) @ _exact_form(*s["b"], case["k"]).t().contiguous()
        return out if s["add"] is None else out + s["add"].double()
    if op == "linear":
        return _exact_values(s["x"]) @ _exact_form(*s["w"], case["k"]).t().contiguous()
    if op == "train":
        draws = _exact_draws(case["tokens"], case["outputs"], seed)
        x, w, dy = s["x"], s["w"], s["dy"]
        return [_exact_values(x) @ _exact_values(w).t().contiguous(),
                _exact_values(dy, draws) @ _exact_values(w.t()).t().contiguous(),
                _exact_values(dy.t(), draws.t()) @ _exact_values(x.t()).t().contiguous()]
    tau, vocab = case["temperature"], case["vocab"]
    losses, gradients = [], []
    for first in range(0, case["rows"], 256):               # 256 rows at a time: fp64 takes room
        part = slice(first, first + 256)
        z, ids, t, grad = s["z"][part].double() / tau, s["ids"][part].long(), s["t"][part].double() / tau, s["grad"][part].double()
        there = (ids >= 0) & (ids < vocab)
        any_there = there.any(dim=1)
        p = torch.softmax(torch.where(there, t, -math.inf), dim=1)
        p = torch.where(any_there.view(-1, 1), p, 0.0)
        lse = torch.logsumexp(z, dim=1)
        place = torch.where(there, ids, 0)
        log_q = z.gather(1, place) - lse.view(-1, 1)
        losses.append(tau ** 2 * torch.where(there & (p > 0), p * (torch.log(p) - log_q), 0.0).sum(dim=1))
        teacher = torch.zeros_like(z).scatter_add_(1, place, p)
        dz = tau * grad.view(-1, 1) * (torch.exp(z - lse.view(-1, 1)) - teacher)
        gradients.append(torch.where(any_there.view(-1, 1), dz, 0.0))
    return [torch.cat(losses), torch.cat(gradients)]
