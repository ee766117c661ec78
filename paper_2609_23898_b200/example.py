"""A data-parallel training step put together: N logical workers train one small network.

Two networks: two linear layers (Job), and a small model of tokens (TokenJob) with the other layers that have weights: an
embedding, norms of queries and keys with the rotation by position, and a gated feed-forward block (layers.Embed, HeadNorm, Gated).

Every worker runs the forward and backward pass of two linear layers on its own batch with 8-bit products
(training.linear, training.linear_backward), which add the weight gradients to its slice of the vector that is
aggregated; the ring (cerar.Plan.allreduce_sim) leaves every worker an approximation of the mean; one worker's is
clipped by its norm (training.TensorSet.grad_norm) and applied by AdamW with 8-bit states (training.TensorSet.adamw).
Nothing waits for the device inside a step.

  python -m paper_2609_23898_b200.example [--model linear|tokens] [--steps 50] [--workers 4] [--tokens 512] [--width 512] [--state-bits 8]
"""
from __future__ import annotations

import argparse

import torch

from . import cerar, layers, training


class Job:
    """Weights w1 (hidden x width), w2 (width x hidden) and a gain per output, learning what a fixed network of the same
    shape computes.  The loss is half the mean square of the difference."""

    def __init__(self, workers=4, tokens=512, width=512, hidden=1024, state_bits=8, lr=3e-3, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.gen, self.N, self.tokens, self.width, self.lr, self.t = gen, workers, tokens, width, lr, 0

        def normal(*shape, std):
            return torch.empty(*shape, device="cuda").normal_(0.0, std, generator=gen)

        shapes = [(hidden, width), (width, hidden), (width,)]
        self.teacher = [normal(*shapes[0], std=width ** -0.5), normal(*shapes[1], std=hidden ** -0.5)]
        self._set_up([normal(*shapes[0], std=width ** -0.5), normal(*shapes[1], std=hidden ** -0.5), torch.ones(width, device="cuda")], state_bits)

    def _set_up(self, master, state_bits):
        """Parameters, the workers' gradients, the ring and the optimizer; vectors do not decay."""
        workers, shapes = self.N, [tuple(p.shape) for p in master]
        self.master, self.params = master, [p.bfloat16() for p in master]
        # every worker's gradients end to end in one vector, zeros up to a length that the ring likes; and the decoded means
        sizes = [p.numel() for p in self.params]
        c = 2 * workers
        self.plan = cerar.Plan.create(workers, c, cerar.EPSILON, 1e-2)
        self.d = self.plan.padded_length(sum(sizes))
        self.grads = torch.zeros(workers, self.d, device="cuda")
        self.means = torch.empty(workers, self.d, device="cuda")
        self.ws = torch.empty(self.plan.workspace_bytes(self.d) // 4, device="cuda")
        starts = [sum(sizes[:i]) for i in range(len(sizes))]
        self.slices = [[g[a:a + n].view(s) for a, n, s in zip(starts, sizes, shapes)] for g in self.grads]
        self.ops = training.Ops()
        self.set = training.TensorSet(self.ops, grads=[self.means[0][a:a + n] for a, n in zip(starts, sizes)], params=self.params,
                                      masters=self.master, state_bits=state_bits,
                                      weight_decay=[0.01 if len(s) > 1 else 0.0 for s in shapes])
        self.clip = torch.empty(3, device="cuda")

    def worker(self, i, w1, w2):
        """One worker's forward and backward pass; returns its loss (on the device)."""
        ops, (g1, g2, gg) = self.ops, self.slices[i]
        x = torch.empty(self.tokens, self.width, device="cuda", dtype=torch.bfloat16).normal_(generator=self.gen)
        target = torch.relu(x.float() @ self.teacher[0].t()) @ self.teacher[1].t()
        h, x_kept = training.linear(ops, x, w1)
        a = torch.relu(h)
        y, a_kept = training.linear(ops, a, w2)
        gain = self.params[2].float()
        err = (y.float() * gain - target) / target.numel()
        gg.copy_((err * y.float()).sum(0))
        da = training.linear_backward(ops, (err * gain).bfloat16(), a_kept, w2, g2, accumulate=False)
        training.linear_backward(ops, da * (h > 0), x_kept, w1, g1, accumulate=False, need_dx=False)
        return 0.5 * err.square().sum() * target.numel()

    def gradients(self):
        """Every worker's forward and backward pass, into its slice; returns their losses."""
        w1, = self.ops.quantize(self.params[0], training.BY_BLOCK)
        w2, = self.ops.quantize(self.params[1], training.BY_BLOCK)
        return [self.worker(i, w1, w2) for i in range(self.N)]

    def step(self):
        """One step of all workers; returns the mean loss (on the device)."""
        self.t += 1
        losses = self.gradients()
        s = torch.cuda.current_stream().cuda_stream
        self.plan.allreduce_sim(self.grads, self.d, self.means, self.d, self.ws, self.d, 1.0 / self.N, s)
        self.set.grad_norm(1.0, out=self.clip)
        self.set.adamw(lr=self.lr, step=self.t, clip=self.clip, seed=self.t)
        return torch.stack(losses).mean()

    def check(self):
        """Waits; raises if a kernel of the ring or of the operators gave up on a wait."""
        self.plan.device_status(torch.cuda.current_stream().cuda_stream)
        self.ops.status()


def _rms(x):
    """x over its root mean square, in the last dimension."""
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class TokenJob(Job):
    """One block of a model of tokens, learning a fixed sequence rule (a token follows from the one before).  Attention itself is made of torch
    operations; every layer with weights adds their gradients to the worker's slice of the aggregated vector."""

    def __init__(self, workers=4, sequences=4, length=128, width=256, heads=4, kv_heads=2, hidden=512, vocab=512, state_bits=8, lr=3e-3, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.gen, self.N, self.lr, self.t = gen, workers, lr, 0
        self.sequences, self.length, self.vocab = sequences, length, vocab
        self.heads, self.kv_heads, self.dim = heads, kv_heads, width // heads
        self.follows = torch.randperm(vocab, device="cuda", generator=gen)

        def normal(*shape, std):
            return torch.empty(*shape, device="cuda").normal_(0.0, std, generator=gen)

        ones = [torch.ones(self.dim, device="cuda") for _ in range(2)]
        self._set_up([normal(vocab, width, std=width ** -0.5), normal((heads + 2 * kv_heads) * self.dim, width, std=width ** -0.5), *ones,
                      normal(width, width, std=width ** -0.5), normal(2 * hidden, width, std=width ** -0.5), normal(width, hidden, std=hidden ** -0.5),
                      normal(vocab, width, std=width ** -0.5)], state_bits)
        self.scale = width ** 0.5
        self.table = layers.rotation_table(self.ops, length, self.dim)
        later = torch.ones(length, length, dtype=torch.bool, device="cuda").triu(1)
        self.mask = torch.zeros(length, length, device="cuda").masked_fill_(later, float("-inf"))

    def batch(self):
        """Token ids (sequences, length + 1)."""
        ids = [torch.randint(self.vocab, (self.sequences,), device="cuda", generator=self.gen)]
        for _ in range(self.length):
            ids.append(self.follows[ids[-1]])
        return torch.stack(ids, 1)

    def worker(self, i, ids, quantized, seen=None):
        """One worker's pass; its loss.  seen: a dict that gets the layers' inputs and outputs."""
        ops, g = self.ops, self.slices[i]
        embedding, _, wq, wk, _, w_in, w_out, _ = self.params
        w_qkv, w_o, w_head = quantized
        x = layers.Embed.apply(embedding, ids[:, :-1].contiguous(), ops, g[0], self.scale)
        e = x
        qkv = training.Linear8.apply(_rms(x), w_qkv, ops, g[1]).unflatten(-1, (-1, self.dim))
        q0, k0, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), dim=2)
        q, k = layers.HeadNorm.apply(q0, k0, wq, wk, ops, self.table, None, g[2], g[3])
        share = self.heads // self.kv_heads
        k_all, v_all = k.repeat_interleave(share, 2), v.repeat_interleave(share, 2)
        scores = torch.einsum("bqhd,bkhd->bhqk", q, k_all).float() * self.dim ** -0.5 + self.mask
        mixed = torch.einsum("bhqk,bkhd->bqhd", scores.softmax(-1).to(v.dtype), v_all).flatten(2)
        x = x + training.Linear8.apply(mixed, w_o, ops, g[4])
        n = _rms(x)
        f = layers.Gated.apply(n, w_in, w_out, ops, g[5], g[6])
        logits = training.Linear8.apply(_rms(x + f), w_head, ops, g[7])
        if seen is not None:
            seen.update(ids=ids, embedded=e, q0=q0, k0=k0, q=q, k=k, gated_in=n, gated=f)
            for t in seen.values():
                if t.requires_grad:
                    t.retain_grad()
        loss = torch.nn.functional.cross_entropy(logits.float().flatten(0, 1), ids[:, 1:].flatten())
        loss.backward()
        return loss.detach()

    def gradients(self):
        self.grads.zero_()
        quantized = [self.ops.quantize(self.params[j], training.BY_BLOCK)[0] for j in (1, 4, 7)]
        return [self.worker(i, self.batch(), quantized) for i in range(self.N)]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--model", choices=("linear", "tokens"), default="linear")
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--state-bits", type=int, default=8)
    a = ap.parse_args()
    if a.model == "linear":
        job = Job(a.workers, a.tokens, a.width, 2 * a.width, a.state_bits)
    else:
        job = TokenJob(a.workers, max(1, a.tokens // 128), 128, a.width, hidden=2 * a.width, state_bits=a.state_bits)
    for i in range(a.steps):
        loss = job.step()
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {loss.item():.5f}  gradient norm {job.clip[0].item():.4f}")
    job.check()


if __name__ == "__main__":
    main()
