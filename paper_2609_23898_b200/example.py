"""A data-parallel training step put together: N logical workers train one small network.

Every worker runs the forward and backward pass of two linear layers on its own batch with 8-bit products
(training.linear, training.linear_backward), which add the weight gradients to its slice of the vector that is
aggregated; the ring (cerar.Plan.allreduce_sim) leaves every worker an approximation of the mean; one worker's is
clipped by its norm (training.TensorSet.grad_norm) and applied by AdamW with 8-bit states (training.TensorSet.adamw).
Nothing waits for the device inside a step.

  python -m paper_2609_23898_b200.example [--steps 50] [--workers 4] [--tokens 512] [--width 512] [--state-bits 8]
"""
from __future__ import annotations

import argparse

import torch

from . import cerar, training


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
        self.master = [normal(*shapes[0], std=width ** -0.5), normal(*shapes[1], std=hidden ** -0.5), torch.ones(width, device="cuda")]
        self.params = [p.bfloat16() for p in self.master]
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
                                      masters=self.master, state_bits=state_bits, weight_decay=[0.01, 0.01, 0.0])
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

    def step(self):
        """One step of all workers; returns the mean loss (on the device)."""
        self.t += 1
        w1, = self.ops.quantize(self.params[0], training.BY_BLOCK)
        w2, = self.ops.quantize(self.params[1], training.BY_BLOCK)
        losses = [self.worker(i, w1, w2) for i in range(self.N)]
        s = torch.cuda.current_stream().cuda_stream
        self.plan.allreduce_sim(self.grads, self.d, self.means, self.d, self.ws, self.d, 1.0 / self.N, s)
        self.set.grad_norm(1.0, out=self.clip)
        self.set.adamw(lr=self.lr, step=self.t, clip=self.clip, seed=self.t)
        return torch.stack(losses).mean()

    def check(self):
        """Waits; raises if a kernel of the ring or of the operators gave up on a wait."""
        self.plan.device_status(torch.cuda.current_stream().cuda_stream)
        self.ops.status()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--state-bits", type=int, default=8)
    a = ap.parse_args()
    job = Job(a.workers, a.tokens, a.width, 2 * a.width, a.state_bits)
    for i in range(a.steps):
        loss = job.step()
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {loss.item():.5f}  gradient norm {job.clip[0].item():.4f}")
    job.check()


if __name__ == "__main__":
    main()
