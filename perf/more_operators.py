"""Cases of the layers around the 8-bit linear one: embedding lookup and its gradient, norms of queries and keys for
each head with the rotation by position, and the gated feed-forward block, each forward and backward.

`run` computes a case either with the framework's operators (`own`) or in a plain form of elementary torch
operations in binary32; `exact` computes it in 64 bits from the operators' definitions.
"""
import math

import torch

own = False

EPS, BASE = 1e-6, 10000.0


def listed():
    return [
        # lookup: the next tokens of a few sequences; the tokens of a training batch
        {"name": "embed_tokens", "op": "embed", "tokens": 4, "vocab": 32000, "width": 2048, "type": "bf16"},
        {"name": "embed_batch", "op": "embed", "tokens": 65536, "vocab": 131072, "width": 2048, "type": "bf16"},
        # its gradient: added to a binary32 slice of the gradient vector for a short odd batch; written whole for a large one
        {"name": "embed_grad_ragged", "op": "embed_grad", "tokens": 1333, "vocab": 5003, "width": 519, "type": "f32", "add": True},
        {"name": "embed_grad_batch", "op": "embed_grad", "tokens": 65536, "vocab": 131072, "width": 2048, "type": "bf16", "add": False},
        # queries and keys of one new token; of a batch with grouped heads, read where a joint projection left them
        {"name": "head_norm_token", "op": "head_norm", "tokens": 1, "q": 16, "k": 4, "dim": 128, "type": "bf16", "pairs": "halves"},
        {"name": "head_norm_batch", "op": "head_norm", "tokens": 16384, "q": 32, "k": 8, "dim": 128, "type": "bf16", "pairs": "halves"},
        # their gradients: a ragged batch in binary32 with neighbouring pairs, a large one
        {"name": "head_norm_grad_ragged", "op": "head_norm_grad", "tokens": 777, "q": 7, "k": 7, "dim": 80, "type": "f32", "pairs": "neighbours"},
        {"name": "head_norm_grad_batch", "op": "head_norm_grad", "tokens": 16384, "q": 32, "k": 8, "dim": 128, "type": "bf16", "pairs": "halves"},
        # gated block forward: one token against all weights; a batch
        {"name": "gated_token", "op": "gated", "tokens": 1, "width": 2048, "hidden": 8192, "act": "silu"},
        {"name": "gated_batch", "op": "gated", "tokens": 16384, "width": 2048, "hidden": 8192, "act": "silu"},
        # forward and backward with both weight gradients: odd sizes, and a training batch
        {"name": "gated_train_ragged", "op": "gated_train", "tokens": 333, "width": 520, "hidden": 1377, "act": "gelu"},
        {"name": "gated_train_batch", "op": "gated_train", "tokens": 16384, "width": 2048, "hidden": 8192, "act": "silu"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "head_norm", "head_norm_grad", "gated", "gated_train"])
    case = {"op": op}
    if op.startswith("embed"):
        case |= {"tokens": _log(rng, 1, 65536), "vocab": _log(rng, 300, 131072), "width": _log(rng, 50, 2048), "type": rng.choice(["bf16", "f32"])}
        if op == "embed":
            case["tokens"] = min(case["tokens"], 32768)     # (binary32 moves twice as much)
        else:
            case["add"] = rng.random() < 0.5
    elif op.startswith("head_norm"):
        k = _log(rng, 1, 8)
        dim = rng.choice([32, 64, 72, 80, 96, 128, 160])
        type_ = rng.choice(["bf16", "f32"])
        case |= {"tokens": _log(rng, 1, 16384 if type_ == "bf16" and dim <= 128 else 6000), "q": k * rng.choice([1, 2, 3, 4]), "k": k, "dim": dim,
                 "type": type_, "pairs": rng.choice(["halves", "neighbours"])}
    else:
        case |= {"tokens": _log(rng, 1, 16384), "width": _log(rng, 100, 2048), "hidden": _log(rng, 100, 8192), "act": rng.choice(["silu", "gelu"])}
    return case


# ------------------------------------------------------------------------------------------------ inputs


def _normal(shape, std, gen, dtype=torch.float32):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen).to(dtype)


def _type(case):
    return torch.float32 if case.get("type") == "f32" else torch.bfloat16


def _rotations(dim):
    """Cosine and sine of the angles of 32768 positions, worked out in 64 bits: (positions, dim / 2, 2)."""
    freq = BASE ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    angle = torch.arange(32768, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, t, ty = case["op"], case["tokens"], _type(case)
    st = {"case": case}
    if op.startswith("embed"):
        v, d = case["vocab"], case["width"]
        # few tokens make up most of a text: the k-th most frequent one with a probability of about 1 / k
        rank = torch.rand(t, generator=gen, device="cuda", dtype=torch.float64).mul_(math.log(v + 1)).exp_().long().sub_(1).clamp_(0, v - 1)
        st["ids"] = torch.randperm(v, generator=gen, device="cuda")[rank]
        st["scale"] = d ** 0.5
        if op == "embed":
            st["table"] = _normal((v, d), 0.02, gen, ty)
        else:
            st["dy"] = _normal((t, d), 1e-3, gen, ty)
            st["dtable"] = _normal((v, d), 1e-3, gen)
    elif op.startswith("head_norm"):
        q, k, d = case["q"], case["k"], case["dim"]
        qkv = _normal((t, q + 2 * k, d), 1.0, gen, ty)          # what one projection gives: queries, keys and values side by side
        st["q"], st["k"] = qkv[:, :q], qkv[:, q:q + k]
        st["wq"], st["wk"] = (1 + _normal((d,), 0.1, gen)).to(ty), (1 + _normal((d,), 0.1, gen)).to(ty)
        st["table"] = _rotations(d)
        start = torch.randint(0, 32768 - t, (1,), generator=gen, device="cuda")
        st["positions"] = start + torch.arange(t, device="cuda")
        if op == "head_norm_grad":
            st["dq"], st["dk"] = _normal((t, q, d), 1e-3, gen, ty), _normal((t, k, d), 1e-3, gen, ty)
            st["dwq"], st["dwk"] = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    else:
        d, f = case["width"], case["hidden"]
        st["x"] = _normal((t, d), 1.0, gen, ty)
        st["w_in"], st["w_out"] = _normal((2 * f, d), d ** -0.5, gen, ty), _normal((d, f), f ** -0.5, gen, ty)
        if op == "gated_train":
            st["dy"] = _normal((t, d), 1e-3, gen, ty)
            st["dw_in"], st["dw_out"] = torch.zeros_like(st["w_in"]), torch.zeros_like(st["w_out"])
    return st


# ------------------------------------------------------------------------------------------------ plain form


def _rotate(z, c, s, pairs):
    a, b = z.chunk(2, -1) if pairs == "halves" else (z[..., 0::2], z[..., 1::2])
    y = (a * c - b * s, b * c + a * s)
    return torch.cat(y, -1) if pairs == "halves" else torch.stack(y, -1).flatten(-2)


def _plain_head(st, x, w):
    """Normed values, the norm's factor, and the rotation of each token."""
    x = x.float()
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    c, s = st["table"][st["positions"]].unbind(-1)
    return x * r, r, c[:, None], s[:, None], w.float()


def _plain_norm(st, x, w):
    n, _, c, s, wf = _plain_head(st, x, w)
    return _rotate(n * wf, c, s, st["case"]["pairs"]).to(x.dtype)


def _plain_norm_grad(st, dy, x, w):
    n, r, c, s, wf = _plain_head(st, x, w)
    dz = _rotate(dy.float(), c, -s, st["case"]["pairs"])
    dn = dz * wf
    dx = r * (dn - n * (dn * n).mean(-1, keepdim=True))
    return dx.to(x.dtype), (dz * n).sum((0, 1))


def _act(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    c = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * c, c + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5


def _plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "embed":
        return [(st["table"][st["ids"]].float() * st["scale"]).to(st["table"].dtype)]
    if op == "embed_grad":
        g = torch.zeros_like(st["dtable"]).index_add_(0, st["ids"], st["dy"].float()) * st["scale"]
        return [st["dtable"].copy_(st["dtable"] + g if case["add"] else g)]
    if op == "head_norm":
        return [_plain_norm(st, st["q"], st["wq"]), _plain_norm(st, st["k"], st["wk"])]
    if op == "head_norm_grad":
        dq, dwq = _plain_norm_grad(st, st["dq"], st["q"], st["wq"])
        dk, dwk = _plain_norm_grad(st, st["dk"], st["k"], st["wk"])
        return [dq, dk, st["dwq"].copy_(dwq), st["dwk"].copy_(dwk)]
    x, w_in, w_out = st["x"].float(), st["w_in"].float(), st["w_out"].float()
    ty = st["x"].dtype
    g, u = (x @ w_in.t()).chunk(2, 1)
    a, da = _act(g, case["act"])
    h = a * u
    y = (h @ w_out.t()).to(ty)
    if op == "gated":
        return [y]
    dy = st["dy"].float()
    dh = dy @ w_out
    dgu = torch.cat([dh * u * da, dh * a], 1)
    return [y, (dgu @ w_in).to(ty), st["dw_in"].copy_(dgu.t() @ x), st["dw_out"].copy_(dy.t() @ h)]


# ------------------------------------------------------------------------------------------------ the framework's operators

_handles = []


def _ops():
    """The operators' handle, made once, as a program does."""
    if not _handles:
        from paper_2609_23898_b200 import training
        _handles.append(training.Ops())
    return _handles[0]


def _own(st):
    from paper_2609_23898_b200 import layers
    case, op, ops = st["case"], st["case"]["op"], _ops()
    if op == "embed":
        return [layers.embed(ops, st["table"], st["ids"], scale=st["scale"])]
    if op == "embed_grad":
        layers.embed_backward(ops, st["dy"], st["ids"], st["dtable"], scale=st["scale"], accumulate=case["add"])
        return [st["dtable"]]
    if op == "head_norm":
        return list(layers.head_norm(ops, st["q"], st["k"], st["wq"], st["wk"], st["table"], st["positions"], eps=EPS, pairs=case["pairs"]))
    if op == "head_norm_grad":
        dq, dk = layers.head_norm_backward(ops, st["dq"], st["dk"], st["q"], st["k"], st["wq"], st["wk"], st["table"], st["positions"],
                                           dwq=st["dwq"], dwk=st["dwk"], accumulate=False, eps=EPS, pairs=case["pairs"])
        return [dq, dk, st["dwq"], st["dwk"]]
    if op == "gated":
        return [layers.gated(ops, st["x"], st["w_in"], st["w_out"], activation=case["act"])]
    y, kept = layers.gated(ops, st["x"], st["w_in"], st["w_out"], activation=case["act"], keep=True)
    dx = layers.gated_backward(ops, st["dy"], kept, st["w_in"], st["w_out"], st["dw_in"], st["dw_out"], accumulate=False)
    return [y, dx, st["dw_in"], st["dw_out"]]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ cost and definition


def work(case):
    op, t = case["op"], case["tokens"]
    size = 4 if case.get("type") == "f32" else 2
    if op.startswith("embed"):
        v, d = case["vocab"], case["width"]
        if op == "embed":
            return {"bytes": 2 * t * d * size + 8 * t, "flops": t * d}
        # rows that some token names: about sum_k (1 - (1 - p_k)^t) of them; all rows where the gradient is written whole
        p = 1 / (math.log(v + 1))
        rows = sum(1 - math.exp(-t * p / k) for k in range(1, v + 1)) if case["add"] else v
        return {"bytes": int(t * d * size + 8 * t + rows * d * 4 * (2 if case["add"] else 1)), "flops": t * d}
    if op.startswith("head_norm"):
        n, d = t * (case["q"] + case["k"]) * case["dim"], case["dim"]
        grad = op == "head_norm_grad"
        return {"bytes": (3 if grad else 2) * n * size + t * (4 * d + 8) + 2 * d * size + (8 * d if grad else 0), "flops": (18 if grad else 8) * n}
    d, f = case["width"], case["hidden"]
    if op == "gated":
        return {"bytes": 4 * t * d + 6 * d * f, "flops": 6 * t * d * f}
    return {"bytes": 8 * t * d + 12 * d * f, "flops": 18 * t * d * f}


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        return [torch.index_select(st["table"], 0, st["ids"]).double() * st["scale"]]
    if op == "embed_grad":
        # sorted by token, then differences of running sums at the ends of each token's run
        order = torch.argsort(st["ids"], stable=True)
        ids = st["ids"][order]
        out = st["dtable"].double() if case["add"] else torch.zeros_like(st["dtable"], dtype=torch.float64)
        runs = torch.cumsum(st["dy"][order].double(), 0)
        last = torch.cat([ids[1:] != ids[:-1], torch.ones(1, dtype=torch.bool, device="cuda")]).nonzero().squeeze(1)
        ends = runs[last]
        ends[1:] -= runs[last[:-1]]
        out[ids[last]] += ends * st["scale"]
        return [out]
    if op.startswith("head_norm"):
        d, h = case["dim"], case["dim"] // 2
        # the rotation as a matrix per token: pairs as complex numbers
        turn = torch.view_as_complex(st["table"][st["positions"]].double().contiguous())[:, None]

        def pairs_of(z):
            z = z.unflatten(-1, (2, h)).transpose(-1, -2) if case["pairs"] == "halves" else z.unflatten(-1, (h, 2))
            return torch.view_as_complex(z.contiguous())

        def back(c):
            z = torch.view_as_real(c)
            return (z.transpose(-1, -2) if case["pairs"] == "halves" else z).flatten(-2)

        out, dws = [], []
        for x, w, dy in ((st["q"], st["wq"], st.get("dq")), (st["k"], st["wk"], st.get("dk"))):
            x, w = x.double(), w.double()
            norm = (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / d + EPS).sqrt()
            if dy is None:
                out.append(back(pairs_of(x / norm * w) * turn))
                continue
            dz = back(pairs_of(dy.double()) * turn.conj())
            dws.append((dz * x / norm).sum((0, 1)))
            out.append(dz * w / norm - x * (dz * w * x).sum(-1, keepdim=True) / (d * norm ** 3))
        return out + dws
    x, w_in, w_out, f = st["x"].double(), st["w_in"].double(), st["w_out"].double(), case["hidden"]
    g, u = x @ w_in[:f].T, x @ w_in[f:].T
    if case["act"] == "silu":
        s = torch.sigmoid(g)
        a, da = g * s, s + g * s * (1 - s)
    else:
        s = torch.special.ndtr(g)
        a, da = g * s, s + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    y = (a * u) @ w_out.T
    if op == "gated":
        return [y]
    dy = st["dy"].double()
    dh = dy @ w_out
    dg, du = dh * u * da, dh * a
    return [y, dg @ w_in[:f] + du @ w_in[f:], torch.cat([dg.T @ x, du.T @ x]), dy.T @ (a * u)]
