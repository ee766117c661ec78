"""Cases of the training-step operators: 8-bit products with a scale per 128 values, the conversion of their
operands, the gradient norm and the AdamW step over many tensors.

`run` computes a case either with the framework's operators (`own`) or in a plain form of elementary torch
operations in binary32; `exact` computes it in 64 bits from the operators' definitions.
"""
import math

import torch

own = False

BLOCK = 128          # values that share a scale in an 8-bit matrix
STATE_BLOCK = 256    # values that share a scale in an 8-bit optimizer state
LR, BETA1, BETA2, EPS, DECAY, STEP, MAX_NORM, SEED = 1e-4, 0.9, 0.95, 1e-8, 0.1, 100, 1.0, 20260923


def listed():
    return [
        # conversion: the activations of one token, and those of eight sequences in both directions at once, as the
        # forward pass does it when it keeps the second copy for the weight gradient
        {"name": "quantize_token", "op": "quantize", "rows": 1, "cols": 2048, "type": "bf16", "row": True, "col": False},
        {"name": "quantize_both", "op": "quantize", "rows": 16384, "cols": 2048, "type": "bf16", "row": True, "col": True},
        # products: one token against a weight matrix, a ragged one with scales that are no powers of two, a large one
        {"name": "product_token", "op": "product", "m": 1, "n": 8192, "k": 2048, "out": "bf16", "b_block": True, "pow2": True},
        {"name": "product_ragged", "op": "product", "m": 333, "n": 1031, "k": 2011, "out": "f32", "b_block": False, "pow2": False},
        {"name": "product_large", "op": "product", "m": 8192, "n": 8192, "k": 8192, "out": "bf16", "b_block": True, "pow2": True},
        # a linear layer's forward and backward pass, conversions included, the weight gradient added to what is there
        {"name": "linear_small", "op": "linear", "m": 256, "n": 1000, "k": 520, "type": "f32"},
        {"name": "linear_large", "op": "linear", "m": 16384, "n": 8192, "k": 2048, "type": "bf16"},
        # gradient norm: a small set, and the parameter count of the framework's largest configuration
        {"name": "norm_small", "op": "norm", "tensors": 16, "total": 65536, "grad": "f32", "packed": False},
        {"name": "norm_large", "op": "norm", "tensors": 292, "total": 1414647808, "grad": "f32", "packed": False},
        # AdamW: a small set in 32 bits (launch latency), the full parameter count in 32 bits, 8-bit states with bf16
        # parameters and master copies, 8-bit states on a ragged set whose gradients lie end to end
        {"name": "adamw_small_32", "op": "adamw", "tensors": 16, "total": 65536, "grad": "f32", "packed": False, "bits": 32, "param": "f32"},
        {"name": "adamw_large_32", "op": "adamw", "tensors": 292, "total": 1414647808, "grad": "f32", "packed": False, "bits": 32, "param": "f32"},
        {"name": "adamw_ragged_8", "op": "adamw", "tensors": 101, "total": 268435456, "grad": "f32", "packed": True, "bits": 8, "param": "master"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "product", "linear", "norm", "adamw"])
    if op == "quantize":
        row = rng.random() < 0.7
        return {"op": op, "rows": _log(rng, 1, 16384), "cols": _log(rng, 100, 8192), "type": rng.choice(["bf16", "f32"]),
                "row": row, "col": not row or rng.random() < 0.5}
    if op == "product":
        return {"op": op, "m": _log(rng, 1, 8192), "n": _log(rng, 100, 8192), "k": _log(rng, 100, 8192),
                "out": rng.choice(["bf16", "f32"]), "b_block": rng.random() < 0.5, "pow2": rng.random() < 0.5}
    if op == "linear":
        return {"op": op, "m": _log(rng, 16, 16384), "n": _log(rng, 128, 8192), "k": _log(rng, 128, 2048),
                "type": rng.choice(["bf16", "f32"])}
    case = {"op": op, "tensors": _log(rng, 1, 300), "total": _log(rng, 30000, 268435456), "grad": rng.choice(["f32", "bf16"]),
            "packed": rng.random() < 0.5}
    if op == "adamw":
        case |= {"bits": rng.choice([32, 8]), "param": rng.choice(["f32", "bf16", "master"])}
    return case


# ------------------------------------------------------------------------------------------------ inputs


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, std, gen, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _activations(rows, cols, type_, gen):
    """Values whose columns differ in size by a factor of a few hundred, as activations and their gradients do."""
    x = _normal((rows, cols), 1.0, gen)
    return x.mul_(torch.exp(_normal((cols,), 1.0, gen))).to(_type(type_))


def _ceil(a, b):
    return -(-a // b)


def _codes(rows, cols, gen):
    """An 8-bit matrix whose rows are a multiple of 16 bytes apart."""
    ld = _ceil(cols, 16) * 16
    return _normal((rows, ld), 60.0, gen).clamp_(-448, 448).to(torch.float8_e4m3fn)[:, :cols]


def _scales(shape, pow2, gen):
    e = torch.randint(-12, -6, shape, generator=gen, device="cuda").float()
    s = torch.exp2(e)
    return s if pow2 else s * (1 + torch.rand(shape, generator=gen, device="cuda"))


def _sizes(case):
    """Element counts of a set: a few large matrices, several smaller ones, many vectors; odd where the total is ragged."""
    n, total = case["tensors"], case["total"]
    weights = [(1.0 if i % 4 == 0 else 0.25 if i % 4 == 1 else 0.001) * (1 + (i * 7 % 5)) for i in range(n)]
    scale = total / sum(weights)
    sizes = [max(1, int(w * scale)) for w in weights]
    sizes[0] = max(1, sizes[0] + total - sum(sizes))
    return sizes


def _layout(case):
    sizes = _sizes(case)
    padded = [_ceil(s, STATE_BLOCK) * STATE_BLOCK for s in sizes]
    starts = [0]
    for p in padded:
        starts.append(starts[-1] + p)
    return sizes, starts


def prepare(case, seed):
    gen = _gen(seed)
    op = case["op"]
    st = {"case": case}
    if own:
        from paper_2609_23898_b200 import training
        st["ops"] = training.Ops()
    if op == "quantize":
        st["x"] = _activations(case["rows"], case["cols"], case["type"], gen)
        return st
    if op == "product":
        m, n, k, kb = case["m"], case["n"], case["k"], _ceil(case["k"], BLOCK)
        st["a"], st["b"] = _codes(m, k, gen), _codes(n, k, gen)
        st["sa"] = _scales((kb, m), case["pow2"], gen)
        st["sb"] = _scales((_ceil(n, BLOCK), kb) if case["b_block"] else (kb, n), case["pow2"], gen)
        if own:
            st["A"] = training.Quantized(st["a"], st["sa"], training.BY_ROW)
            st["B"] = training.Quantized(st["b"], st["sb"], training.BY_BLOCK if case["b_block"] else training.BY_ROW)
        return st
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        st["x"] = _activations(m, k, case["type"], gen)
        st["w"] = _normal((n, k), k ** -0.5, gen).to(_type(case["type"]))
        st["dy"] = _activations(m, n, case["type"], gen).mul_(1e-3)
        st["dw"] = _normal((n, k), 1e-2, gen)
        return st
    # a set of tensors, each starting at a multiple of 256 elements; states lie the same way
    sizes, starts = _layout(case)
    total = starts[-1]
    live = None
    if any(s % STATE_BLOCK for s in sizes):
        live = torch.zeros(total, dtype=torch.bool, device="cuda")
        for s, a in zip(sizes, starts):
            live[a:a + s] = True
    grad = _normal((total,), 1e-3, gen, _type(case["grad"]))
    if live is not None:
        grad *= live
    if case["packed"]:  # gradients end to end, as one aggregated vector holds them
        if live is None:
            live = torch.ones(total, dtype=torch.bool, device="cuda")
        st["where"] = live.nonzero().squeeze(1)
        grad = grad[live]
        first = [0]
        for s in sizes:
            first.append(first[-1] + s)
    else:
        first = starts
    st["grad"], st["total"] = grad, total
    grads = [grad[a:a + s] for a, s in zip(first, sizes)]
    if op == "norm":
        if own:
            st["set"] = training.TensorSet(st["ops"], grads=grads)
        return st
    st["clip"] = torch.tensor([2.0, 0.5, 1.0], device="cuda")
    p = _normal((total,), 0.02, gen)
    if live is not None:
        p *= live
    st["param"] = p if case["param"] == "f32" else p.bfloat16()
    st["master"] = p if case["param"] == "master" else None
    m = _normal((total,), 3e-4, gen)
    v = torch.empty(total, device="cuda").exponential_(1.0, generator=gen).mul_(2.5e-7)
    if live is not None:
        m *= live
        v *= live
    if case["bits"] == 8:
        nb = total // STATE_BLOCK
        m, r = m.view(nb, STATE_BLOCK), v.sqrt_().view(nb, STATE_BLOCK)
        st["m_scale"] = _pow2_scale(m.abs().amax(1), 448.0)
        st["v_scale"] = _pow2_scale(r.amax(1), 448.0)
        m = (m / st["m_scale"][:, None]).to(torch.float8_e4m3fn).view(-1)
        v = (r / st["v_scale"][:, None]).to(torch.float8_e4m3fn).view(-1)
    st["m"], st["v"] = m, v
    # matrices (the first tensor of every four and the one after it) decay, the vectors do not
    decays = [DECAY if i % 4 < 2 else 0.0 for i in range(len(sizes))]
    if own:
        st["set"] = training.TensorSet(
            st["ops"], params=[st["param"][a:a + s] for a, s in zip(starts, sizes)], grads=grads,
            masters=None if st["master"] is None else [st["master"][a:a + s] for a, s in zip(starts, sizes)],
            weight_decay=decays, state_bits=case["bits"], m=st["m"], v=st["v"], m_scale=st.get("m_scale"), v_scale=st.get("v_scale"))
    else:
        counts = torch.tensor([b - a for a, b in zip(starts, starts[1:])], device="cuda")
        st["decay"], st["counts"] = torch.tensor(decays, device="cuda"), counts
    return st


# ------------------------------------------------------------------------------------------------ plain form


def _pow2_scale(amax, top):
    """2^e with the smallest e that brings amax to top or below, 1 for a maximum of zero."""
    frac, e = torch.frexp(amax)
    top_frac, top_e = math.frexp(top)
    e = (e - top_e + (frac > top_frac)).clamp(-100, 100)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.ones_like(amax))


def _plain_quantize(x, rows, cols):
    """Codes (as values) and scales of x with a scale per rows x cols values."""
    r, c = x.shape
    x = x.float()
    pad = torch.nn.functional.pad(x, (0, -c % cols, 0, -r % rows)).view(_ceil(r, rows), rows, _ceil(c, cols), cols)
    scale = _pow2_scale(pad.abs().amax((1, 3)), 448.0)
    q = (pad / scale[:, None, :, None]).to(torch.float8_e4m3fn).view(_ceil(r, rows) * rows, -1)[:r, :c]
    return q, scale


def _expand(scale, rows, cols, shape):
    return scale.repeat_interleave(rows, 0)[:shape[0]].repeat_interleave(cols, 1)[:, :shape[1]]


def _plain_value(x, rows, cols):
    q, scale = _plain_quantize(x, rows, cols)
    return q.float() * _expand(scale, rows, cols, q.shape)


def _mix(block, seed, total):
    """32 random bits for each of `total` elements, from the element's place and the seed."""
    mask = 0xFFFFFFFF
    nb = total // STATE_BLOCK
    key = torch.arange(nb, dtype=torch.int64, device="cuda")
    key = ((key & mask) * 0x9E3779B1 + ((key >> 32) + 1) * 0x7FEB352D + seed * 0x85157AF5 + block * 0x632BE5AB) & mask
    key = _scramble(key)
    lane = torch.arange(STATE_BLOCK, dtype=torch.int64, device="cuda") * 0x9E3779B9
    return _scramble((key[:, None] + lane[None, :]) & mask).view(-1)


def _scramble(h):
    mask = 0xFFFFFFFF
    h = ((h ^ (h >> 16)) * 0x7FEB352D) & mask
    h = ((h ^ (h >> 15)) * 0x846CA68B) & mask
    return h ^ (h >> 16)


def _to_bf16_random(x, bits16):
    """binary32 to bfloat16, up with the probability of the part that is cut off."""
    return (((x.view(torch.int32).long() + bits16) >> 16) << 16).to(torch.int32).view(torch.float32).bfloat16()


def _to_8_random(y, bits16):
    """Codes of 0 <= y <= 448 (four exponent and three mantissa bits), up with the probability of the part that is cut
    off; after the product the code is the exponent and the first mantissa bits of the binary32 number."""
    return ((y * 2.0 ** -120).view(torch.int32) + ((bits16 << 4) + 8)) >> 20


def _plain_adamw(st):
    case = st["case"]
    total = st["total"]
    g = st["grad"].float()
    if case["packed"]:
        full = torch.zeros(total, device="cuda")
        full[st["where"]] = g
        g = full
    nb = total // STATE_BLOCK
    if case["bits"] == 8:
        m = (st["m"].float().view(nb, -1) * st["m_scale"][:, None]).view(-1)
        v = (st["v"].float().view(nb, -1) * st["v_scale"][:, None]).square().view(-1)
    else:
        m, v = st["m"], st["v"]
    g = g * st["clip"][1]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g.square() * (1 - BETA2)
    r = v.sqrt()
    keep = (1 - LR * st["decay"]).repeat_interleave(st["counts"])
    p = (st["param"] if st["master"] is None else st["master"]).float()
    p = p * keep - LR / (1 - BETA1 ** STEP) * m / (r * (1 - BETA2 ** STEP) ** -0.5 + EPS)
    if case["bits"] == 32:
        st["m"].copy_(m)
        st["v"].copy_(v)
    if case["bits"] == 8:
        bits = _mix(0, SEED, total)
        m, r = m.view(nb, -1), r.view(nb, -1)
        ms, rs = _pow2_scale(m.abs().amax(1), 448.0), _pow2_scale(r.amax(1), 448.0)
        y = (m / ms[:, None]).view(-1)
        st["m"].view(torch.uint8).copy_(_to_8_random(y.abs(), bits >> 16) + (y < 0) * 128)
        y = (r / rs[:, None]).view(-1)
        c = _to_8_random(y, bits & 0xFFFF)
        st["v"].view(torch.uint8).copy_(torch.where(y > 0, c.clamp(min=1), c))
        st["m_scale"].copy_(ms)
        st["v_scale"].copy_(rs)
    if case["param"] == "bf16":
        st["param"].copy_(_to_bf16_random(p, _mix(1, SEED, total) >> 16))
    else:
        st["param"].copy_(p)
        if st["master"] is not None:
            st["master"].copy_(p)


def _plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "quantize":
        out = []
        if case["row"]:
            q, s = _plain_quantize(st["x"], 1, BLOCK)
            out += [q, s.t()]
        if case["col"]:
            out += list(_plain_quantize(st["x"], BLOCK, 1))
        return out
    if op == "product":
        a = st["a"].float() * _expand(st["sa"].t(), 1, BLOCK, st["a"].shape)
        b = st["b"].float() * (_expand(st["sb"], BLOCK, BLOCK, st["b"].shape) if case["b_block"] else _expand(st["sb"].t(), 1, BLOCK, st["b"].shape))
        return (a @ b.t()).to(_type(case["out"]))
    if op == "linear":
        w = _plain_value(st["w"], BLOCK, BLOCK)
        t = st["x"].dtype
        y = (_plain_value(st["x"], 1, BLOCK) @ w.t()).to(t)
        dx = (_plain_value(st["dy"], 1, BLOCK) @ w).to(t)
        st["dw"] += _plain_value(st["dy"], BLOCK, 1).t() @ _plain_value(st["x"], BLOCK, 1)
        return [y, dx, st["dw"]]
    if op == "norm":
        norm = st["grad"].float().square().sum().sqrt()
        return torch.stack([norm, (MAX_NORM / (norm + 1e-6)).clamp(max=1.0), torch.isfinite(norm).float()])
    _plain_adamw(st)
    return _adamw_outputs(st)


def _adamw_outputs(st):
    """Parameters and states; states in 8 bits (of the first moment and of the second one's root) with their scales."""
    out = [st["param"], st["m"], st["v"]]
    if st["case"]["bits"] == 8:
        out += [st["m_scale"], st["v_scale"]]
    return out if st["master"] is None else [*out, st["master"]]


# ------------------------------------------------------------------------------------------------ one pass


def run(st):
    if not own:
        return _plain(st)
    from paper_2609_23898_b200 import training as T
    case, op, ops = st["case"], st["case"]["op"], st["ops"]
    if op == "quantize":
        how = [T.BY_ROW] * case["row"] + [T.BY_COLUMN] * case["col"]
        return [t for q in ops.quantize(st["x"], *how) for t in (q.codes, q.scales)]
    if op == "product":
        return ops.matmul(st["A"], st["B"], trans_b=True, dtype=_type(case["out"]))
    if op == "linear":
        t = st["x"].dtype
        xr, xc = ops.quantize(st["x"], T.BY_ROW, T.BY_COLUMN)
        w, = ops.quantize(st["w"], T.BY_BLOCK)
        y = ops.matmul(xr, w, trans_b=True, dtype=t)
        dr, dc = ops.quantize(st["dy"], T.BY_ROW, T.BY_COLUMN)
        dx = ops.matmul(dr, w, dtype=t)
        ops.matmul(dc, xc, trans_a=True, out=st["dw"], accumulate=True)
        return [y, dx, st["dw"]]
    if op == "norm":
        return st["set"].grad_norm(MAX_NORM)
    st["set"].adamw(lr=LR, betas=(BETA1, BETA2), eps=EPS, step=STEP, clip=st["clip"], seed=SEED)
    return _adamw_outputs(st)


def work(case):
    op = case["op"]
    size = {"f32": 4, "bf16": 2}
    if op == "quantize":
        n, outs = case["rows"] * case["cols"], case["row"] + case["col"]
        return {"bytes": n * (size[case["type"]] + outs * (1 + 4 / BLOCK)), "flops": 0}
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * k + m * n * size[case["out"]], "flops": 2 * m * n * k}
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        b = size[case["type"]]
        return {"bytes": (2 * m * k + 2 * m * n + n * k) * b + 8 * n * k, "flops": 6 * m * n * k}
    total, g = case["total"], size[case["grad"]]
    if op == "norm":
        return {"bytes": total * g, "flops": 2 * total}
    p = {"f32": 8, "bf16": 4, "master": 10}[case["param"]]
    s = 16 if case["bits"] == 32 else 4 + 16 / STATE_BLOCK
    return {"bytes": total * (g + p + s), "flops": 15 * total}


# ------------------------------------------------------------------------------------------------ 64 bits


def _scale64(amax, top):
    e = torch.ceil(torch.log2(amax / top)).clamp(-100, 100)
    e = torch.where(amax <= top * torch.exp2(e - 1), e - 1, e)  # the logarithm may be a bit high or low
    e = torch.where(amax > top * torch.exp2(e), e + 1, e).clamp(-100, 100)
    return torch.where(amax > 0, torch.exp2(e), torch.ones_like(amax))


def _step64(y, mantissa, low):
    """Distance of neighbouring codes at |y|: `mantissa` bits, 2^low below the normal numbers."""
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -60)))
    return torch.exp2((e - mantissa).clamp(min=low))


def _quantize64(x, rows, cols):
    r, c = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -c % cols, 0, -r % rows))
    tiles = x.unflatten(0, (-1, rows)).unflatten(2, (-1, cols))
    scale = _scale64(tiles.abs().amax(3).amax(1), 448.0)
    wide = torch.kron(scale, torch.ones(rows, cols, dtype=torch.float64, device=x.device))
    y = x / wide
    d = _step64(y, 3, -9)
    return (torch.round(y / d) * d)[:r, :c], scale, wide[:r, :c]


def _value64(x, rows, cols):
    q, _, wide = _quantize64(x, rows, cols)
    return q * wide


def _bits64(stream, total):
    """The random numbers of the rounding, an input of the operator: whole numbers in 32 bits."""
    return _mix(stream, SEED, total)


def _exact_adamw(st, case):
    total = st["total"]
    nb = total // STATE_BLOCK
    g = torch.zeros(total, dtype=torch.float64, device="cuda")
    if case["packed"]:
        g[st["where"]] = st["grad"].double()
    else:
        g += st["grad"]
    if case["bits"] == 8:
        m = st["m"].double() * st["m_scale"].double().repeat_interleave(STATE_BLOCK)
        v = (st["v"].double() * st["v_scale"].double().repeat_interleave(STATE_BLOCK)) ** 2
    else:
        m, v = st["m"].double(), st["v"].double()
    g *= 0.5
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    del g
    p = (st["param"] if st["master"] is None else st["master"]).double()
    p = p - LR * torch.repeat_interleave(st["decay"].double(), st["counts"]) * p
    p = p - LR * (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS)
    if case["param"] == "bf16":
        d = torch.exp2(torch.floor(torch.log2(p.abs().clamp(min=2.0 ** -120))) - 7)
        q = torch.sign(p) * torch.floor(p.abs() / d + (_bits64(1, total) >> 16).double() / 65536) * d
    else:
        q = p
    if case["bits"] == 32:
        return [q, m, v] + ([p] if case["param"] == "master" else [])
    bits = _bits64(0, total)
    ms = _scale64(m.view(nb, -1).abs().amax(1), 448.0)
    y = m / ms.repeat_interleave(STATE_BLOCK)
    d = _step64(y, 3, -9)
    m = torch.sign(y) * torch.floor(y.abs() / d + ((bits >> 16).double() + 0.5) / 65536) * d
    r = torch.sqrt(v)
    rs = _scale64(r.view(nb, -1).amax(1), 448.0)
    y = r / rs.repeat_interleave(STATE_BLOCK)
    d = _step64(y, 3, -9)
    r = torch.floor(y / d + ((bits & 0xFFFF).double() + 0.5) / 65536) * d
    r = torch.where(y > 0, r.clamp(min=2.0 ** -9), r)
    return [q, m, r, ms, rs] + ([p] if case["param"] == "master" else [])


def exact(case, seed):
    op = case["op"]
    if op == "adamw" and case["total"] > 300_000_000:
        return None  # the double-precision copies of such a set do not fit beside its state
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if op == "quantize":
        out = []
        if case["row"]:
            q, s, _ = _quantize64(st["x"], 1, BLOCK)
            out += [q, s.t()]
        if case["col"]:
            q, s, _ = _quantize64(st["x"], BLOCK, 1)
            out += [q, s]
        return out
    if op == "product":
        ones = torch.ones(1, BLOCK, dtype=torch.float64, device="cuda")
        a = st["a"].double() * torch.kron(st["sa"].double().t().contiguous(), ones)[:, :case["k"]]
        if case["b_block"]:
            b = torch.kron(st["sb"].double(), ones.expand(BLOCK, -1).contiguous())[:case["n"], :case["k"]]
        else:
            b = torch.kron(st["sb"].double().t().contiguous(), ones)[:, :case["k"]]
        return a @ (b * st["b"].double()).t()
    if op == "linear":
        w = _value64(st["w"], BLOCK, BLOCK)
        y = _value64(st["x"], 1, BLOCK) @ w.t()
        dx = _value64(st["dy"], 1, BLOCK) @ w
        dw = st["dw"].double() + _value64(st["dy"], BLOCK, 1).t() @ _value64(st["x"], BLOCK, 1)
        return [y, dx, dw]
    if op == "norm":
        norm = math.sqrt(sum(float(c.double().square().sum()) for c in st["grad"].split(1 << 26)))
        return torch.tensor([norm, min(1.0, MAX_NORM / (norm + 1e-6)), 1.0], dtype=torch.float64, device="cuda")
    return _exact_adamw(st, case)
