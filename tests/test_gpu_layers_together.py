"""The layers as they are used together: a training step of the example's model of tokens, embedding, head norms and gated block beside the
8-bit linear layers, all weight gradients in the aggregated vector.  On the GPU.

What every layer of these put into the vector is the formula's, in 64 bits, on the inputs and the output gradients that autograd handed it.  Tolerances
as in the layers' own tests: the embedding's sum of n binary32 values within (n + 4) 2^-24 of the sum of their magnitudes; head norms (n + d / 2 + 12)
2^-24 of it; the block's operands are rounded to bfloat16 (2^-8 of themselves) behind an activation and a product, three times at most along any
term, and sums add 2^-23 (264 + K / 4096): 2^-6 of the sum of magnitudes holds them all.
"""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_of_all_workers(bits):
    import torch
    from paper_2609_23898_b200 import example
    job = example.TokenJob(workers=4, sequences=2, length=48, width=128, heads=4, kv_heads=2, hidden=200, vocab=130, state_bits=bits)
    before = [p.clone() for p in job.params]
    for _ in range(3):
        loss = job.step()
    job.check()
    assert bool(torch.isfinite(loss)) and job.clip[2].item() == 1
    assert all(not torch.equal(a, b) for a, b in zip(before, job.params))
    exact = job.grads.double().mean(0)
    for i in range(4):
        assert ((job.means[i].double() - exact).norm() / exact.norm()).item() < 0.1        # (the design's error, eps = 1e-2, below 10 eps)


def test_the_gradients_are_the_formulas():
    import torch
    from paper_2609_23898_b200 import example, training
    job = example.TokenJob(workers=2, sequences=3, length=40, width=128, heads=4, kv_heads=2, hidden=136, vocab=70)
    job.grads.zero_()
    quantized = [job.ops.quantize(job.params[j], training.BY_BLOCK)[0] for j in (1, 4, 7)]
    seen = {}
    job.worker(1, job.batch(), quantized, seen)
    assert not bool(job.grads[0].any())
    g = job.slices[1]
    assert all(bool(t.any()) for t in g)
    # embedding
    ids, dy = seen["ids"][:, :-1].flatten(), seen["embedded"].grad.flatten(0, 1).double()
    want = torch.zeros(job.vocab, dy.size(1), dtype=torch.float64, device="cuda").index_add_(0, ids, dy) * job.scale
    size = torch.zeros_like(want).index_add_(0, ids, dy.abs()) * job.scale
    n = torch.bincount(ids, minlength=job.vocab)[:, None]
    assert bool(((g[0].double() - want).abs() <= size * (n + 4) * U * 1.01).all())
    # head norms
    d = job.dim
    c, s = job.table.double().unbind(-1)
    c, s = torch.cat((c, c), -1)[:, None], torch.cat((s, s), -1)[:, None]
    for x, y, w, dw in (("q0", "q", 2, g[2]), ("k0", "k", 3, g[3])):
        x, dy = seen[x].detach().double(), seen[y].grad.double()
        other = torch.cat((dy[..., d // 2:], -dy[..., :d // 2]), -1)
        r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        want, size = ((dy * c + other * s) * x * r).sum((0, 1, 2)), ((dy.abs() + other.abs()) * (x * r).abs()).sum((0, 1, 2))
        assert bool(((dw.double() - want).abs() <= size * (x[..., 0].numel() + d / 2 + 12) * U).all())
    # gated block
    w_in, w_out, x, dy = job.params[5].double(), job.params[6].double(), seen["gated_in"].detach().flatten(0, 1).double(), seen["gated"].grad.flatten(0, 1).double()
    f = w_out.size(1)
    a, u = x @ w_in[:f].t(), x @ w_in[f:].t()
    sg = torch.sigmoid(a)
    act, slope = a * sg, sg * (1 + a * (1 - sg))
    dh, mag = dy @ w_out, dy.abs() @ w_out.abs()
    ma, mu = x.abs() @ w_in[:f].abs().t(), x.abs() @ w_in[f:].abs().t()
    for got, want, size in ((g[5], torch.cat(((dh * u * slope).t() @ x, (dh * act).t() @ x)), torch.cat(((mag * mu * 1.2).t() @ x.abs(), (mag * ma).t() @ x.abs()))),
                            (g[6], dy.t() @ (act * u), dy.abs().t() @ (ma * mu))):
        assert bool(((got.double() - want).abs() <= 2.0 ** -6 * size).all())
        assert float((got.double() - want).norm() / want.norm()) < 2.0 ** -6


def test_two_streams_and_a_graph():
    """Forward and backward passes of all three on two streams at a time, and captured once and replayed: the same bits."""
    import torch
    from paper_2609_23898_b200 import layers, training
    ops = training.Ops()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def normal(*s, std=1.0):
        return torch.randn(*s, device="cuda", generator=g) * std

    table, w_in, w_out = normal(300, 64).bfloat16(), normal(160, 64, std=0.1).bfloat16(), normal(64, 80, std=0.1).bfloat16()
    w, rot = normal(16).bfloat16(), layers.rotation_table(ops, 600, 16)
    sets = [(torch.randint(300, (500,), device="cuda", generator=g), normal(500, 64).bfloat16()) for _ in range(2)]

    def run(ids, dy):
        grads = [torch.zeros(300, 64, device="cuda"), torch.zeros(16, device="cuda"), torch.zeros(160, 64, device="cuda"), torch.zeros(64, 80, device="cuda")]
        x = layers.embed(ops, table, ids)
        q, _ = layers.head_norm(ops, x.view(-1, 4, 16), None, w, None, rot)
        y, kept = layers.gated(ops, q.reshape(-1, 64), w_in, w_out, keep=True)
        dx = layers.gated_backward(ops, dy, kept, w_in, w_out, grads[2], grads[3])
        dq, _ = layers.head_norm_backward(ops, dx.view(-1, 4, 16), None, x.view(-1, 4, 16), None, w, None, rot, dwq=grads[1])
        layers.embed_backward(ops, dq.reshape(-1, 64), ids, grads[0])
        return [y, dx, dq, *grads]

    want = [run(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = run(*sets[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))
    ids, dy = (t.clone() for t in sets[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(ids, dy)
    for k in (1, 0, 1):
        ids.copy_(sets[k][0])
        dy.copy_(sets[k][1])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[k]))
    ops.status()


def test_captured_backward_pass_beside_an_eager_graph():
    """A backward pass captured into a graph while an eager autograd graph through the same layers lives: what autograd follows in place of an input
    belongs to one call (a leaf that both graphs share has torch's own rule against that)."""
    import torch
    from paper_2609_23898_b200 import layers, training
    ops = training.Ops()
    w_in, w_out = torch.randn(96, 32, device="cuda").bfloat16() * 0.2, torch.randn(32, 48, device="cuda").bfloat16() * 0.2
    table, ids, w = torch.randn(50, 32, device="cuda").bfloat16(), torch.randint(50, (20,), device="cuda"), torch.ones(8, device="cuda").bfloat16()
    grads = [torch.zeros(50, 32, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(96, 32, device="cuda"), torch.zeros(32, 48, device="cuda")]

    def loss():
        x = layers.Embed.apply(table, ids, ops, grads[0], 1.0)
        x, _ = layers.HeadNorm.apply(x.view(20, 4, 8), None, w, None, ops, None, None, grads[1])
        return layers.Gated.apply(x.flatten(1), w_in, w_out, ops, grads[2], grads[3]).float().square().sum()

    alive = loss()                                     # lives through the capture
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loss().backward()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss().backward()
    for t in grads:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    first = [t.clone() for t in grads]
    assert all(bool(t.any()) for t in first)
    for t in grads:
        t.zero_()
    alive.backward()
    assert all(torch.equal(a, b) for a, b in zip(first, grads))
    ops.status()


def test_weights_made_in_inference_mode_and_saved_tensor_hooks():
    """Such weights cannot be saved by autograd: they are held; what is saved passes through hooks (here: to the host and back) and comes back the same."""
    import torch
    from paper_2609_23898_b200 import layers, training
    ops = training.Ops()
    with torch.inference_mode():
        frozen = [torch.randn(96, 32, device="cuda").bfloat16() * 0.2, torch.randn(32, 48, device="cuda").bfloat16() * 0.2,
                  torch.randn(50, 32, device="cuda").bfloat16(), torch.ones(8, device="cuda").bfloat16()]
    ids = torch.randint(50, (20,), device="cuda")
    rot = layers.rotation_table(ops, 20, 8)
    results = []
    for weights, hooks in ((frozen, False), ([t.clone() for t in frozen], False), ([t.clone() for t in frozen], True)):
        grads = [torch.zeros(50, 32, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(96, 32, device="cuda"), torch.zeros(32, 48, device="cuda")]

        def run():
            x = layers.Embed.apply(weights[2], ids, ops, grads[0], 1.0)
            x, _ = layers.HeadNorm.apply(x.view(20, 4, 8), None, weights[3], None, ops, rot, None, grads[1])
            return layers.Gated.apply(x.flatten(1), weights[0], weights[1], ops, grads[2], grads[3])

        if hooks:
            with torch.autograd.graph.saved_tensors_hooks(lambda t: t.cpu(), lambda t: t.cuda()):
                y = run()
        else:
            y = run()
        y.backward(torch.ones_like(y))
        results.append(grads)
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
    ops.status()


def test_two_host_threads_and_launch_counts():
    """Handles of their own on two host threads at a time; every launch is counted."""
    import threading
    import torch
    from paper_2609_23898_b200 import layers, training
    table, ids = torch.randn(300, 40, device="cuda"), torch.randint(300, (700,), device="cuda")
    x, w_in, w_out = torch.randn(64, 40, device="cuda").bfloat16(), torch.randn(96, 40, device="cuda").bfloat16(), torch.randn(40, 48, device="cuda").bfloat16()
    torch.cuda.synchronize()
    out, errors = [None, None], []

    def work(i):
        try:
            ops = training.Ops()
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    d = torch.zeros(300, 40, device="cuda")
                    layers.embed_backward(ops, layers.embed(ops, table, ids), ids, d)
                    y = layers.gated(ops, x, w_in, w_out)
                ops.status()
                out[i] = (d, y, ops.launch_count())
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]) and out[0][2] == out[1][2] == 20 * (1 + 3 + 2)
