"""training.Linear8 inside an autograd graph, on the GPU.

Where numbers are compared, inputs are small integers, which the 8-bit format holds exactly with any of its scales, and all sums stay
below 2^24: y, dx and dw are then equal to the layer's formulas y = x w^T, dx = dy w, dw = dy^T x in 64 bits, with no tolerance.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    import torch
    from paper_2609_23898_b200 import training
    assert torch.cuda.is_available()
    o = training.Ops()
    yield o
    o.status()


def whole(rng, *shape):
    import torch
    return torch.from_numpy(rng.integers(-8, 9, shape).astype(np.float32)).cuda()


def layer(ops, rng, n, k):
    from paper_2609_23898_b200 import training as R
    import torch
    w = whole(rng, n, k)
    return w, ops.quantize(w, R.BY_BLOCK)[0], torch.zeros(n, k, device="cuda")


# ---------------------------------------------------------------------------------------------------- strides

def strided(t, how):
    """The same values with other strides: rows not contiguous, a slice of a wider tensor, an element repeated."""
    import torch
    if how == "transposed":
        return t.t().contiguous().t()
    if how == "every second":
        return torch.stack((t, t + 1), -1).flatten(-2)[:, ::2]
    if how == "permuted":
        return t.view(10, -1, t.size(1)).transpose(0, 1).contiguous().transpose(0, 1)
    return t[:1, :1].expand_as(t) if how == "expanded" else t[:1].expand_as(t)


@pytest.mark.parametrize("how", ["transposed", "every second", "permuted", "expanded", "one row"])
def test_inputs_and_gradients_of_any_strides(ops, how):
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(4)
    n, k = 70, 48
    w, wq, dw = layer(ops, rng, n, k)
    x = strided(whole(rng, 60, k), how).requires_grad_()
    dy = strided(whole(rng, 60, n), how)
    y = R.Linear8.apply(x, wq, ops, dw)
    assert y.shape == (*x.shape[:-1], n)
    assert torch.equal(y.detach().double(), x.detach().double() @ w.double().t())
    y.backward(dy)
    x2, d2 = x.detach().double().reshape(-1, k), dy.double().reshape(-1, n)
    assert torch.equal(x.grad.double().reshape(-1, k), d2 @ w.double()) and torch.equal(dw.double(), d2.t() @ x2)


def test_losses_whose_gradient_is_expanded_or_transposed(ops):
    """y.sum() hands back one element with strides 0, a loss on y.t() a transposed gradient."""
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(5)
    w, wq, dw = layer(ops, rng, 70, 48)
    x = whole(rng, 60, 48).requires_grad_()
    R.Linear8.apply(x, wq, ops, dw).sum().backward()
    ones = torch.ones(60, 70, device="cuda", dtype=torch.float64)
    assert torch.equal(x.grad.double(), ones @ w.double()) and torch.equal(dw.double(), ones.t() @ x.detach().double())
    dw.zero_()
    x.grad = None
    v = whole(rng, 60)
    (R.Linear8.apply(x, wq, ops, dw).t().contiguous() @ v).sum().backward()
    dy = v.double()[:, None].expand(60, 70)
    assert torch.equal(x.grad.double(), dy @ w.double()) and torch.equal(dw.double(), dy.t() @ x.detach().double())


@pytest.mark.parametrize("shape,strides", [((0, 200), (0, 0)), ((0, 200), (1, 2)), ((200, 0), (0, 1)), ((200, 0), (0, 0))])
def test_nothing_may_have_any_strides(ops, shape, strides):
    import torch
    from paper_2609_23898_b200 import training as R
    x = torch.empty(8, device="cuda").as_strided(shape, strides)
    for q in [*ops.quantize(x, 0, 1, 2), *ops.quantize(x, 0)]:
        assert tuple(q.shape) == shape and q.dequantize().shape == shape
    w, = ops.quantize(torch.ones(70, shape[1], device="cuda"), R.BY_BLOCK)
    assert torch.equal(R.Linear8.apply(x, w, ops, None), torch.zeros(shape[0], 70, device="cuda"))
    out = torch.empty(8, device="cuda").as_strided((0, 70), strides)
    a, = ops.quantize(torch.empty(0, 200, device="cuda"), R.BY_ROW)
    b, = ops.quantize(torch.ones(70, 200, device="cuda"), R.BY_ROW)
    assert ops.matmul(a, b, trans_b=True, out=out) is out


# ---------------------------------------------------------------------------------------------------- inputs without a gradient

@pytest.mark.parametrize("shape", [(150, 200), (10, 15, 200), (200,), (1, 200), (0, 200)])
def test_weight_gradient_of_a_first_layer(ops, shape):
    """x is data: nothing but what lies above the layer has a gradient of its own, and dw is dy^T x all the same."""
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(len(shape))
    n, k = 70, 200
    x, (w, wq, dw) = whole(rng, *shape), layer(ops, rng, n, k)
    gain = torch.ones(n, device="cuda", requires_grad=True)
    y = R.Linear8.apply(x, wq, ops, dw)
    dy = whole(rng, *y.shape)
    (y * gain * dy).sum().backward()
    want = dy.double().reshape(-1, n).t() @ x.double().reshape(-1, k)
    assert torch.equal(dw.double(), want)
    assert x.grad is None and torch.equal(gain.grad.double(), (dy.double() * (x.double() @ w.double().t())).reshape(-1, n).sum(0))


def test_two_layers_the_first_on_data(ops):
    """Frozen layers below, a ReLU between: both weight gradients are those of the formula."""
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.integers(-2, 3, (130, 40)).astype(np.float32)).cuda()
    (w1, q1, d1), (w2, q2, d2) = layer(ops, rng, 24, 40), layer(ops, rng, 50, 24)
    with torch.no_grad():
        x = x * 1.0                                                        # what a frozen layer hands on
    h = R.Linear8.apply(x, q1, ops, d1)
    a = torch.where(h > 0, 4.0, -1.0) + 0 * h                              # values the format holds; its gradient with respect to h is 0
    y = R.Linear8.apply(a + h.clamp(-8, 8), q2, ops, d2)
    dy = torch.from_numpy(rng.integers(-1, 2, tuple(y.shape)).astype(np.float32)).cuda()
    y.backward(dy)
    hin = (a + h.clamp(-8, 8)).detach().double()
    assert torch.equal(d2.double(), dy.double().t() @ hin)
    dh = (dy.double() @ w2.double()) * ((h >= -8) & (h <= 8))
    # dh is quantized by column for dw1: within 2^-4 of each element or of 2^-17 of its column's largest
    err = (dh.abs() / 16 + dh.abs().amax(0) * 2.0 ** -17).t() @ x.double().abs()
    assert bool(((d1.double() - dh.t() @ x.double()).abs() <= err * 1.01).all()) and bool(d1.any())


def test_frozen_weights_and_frozen_input(ops):
    """Without dw only x has a gradient; with neither, or without gradients enabled, the result has none."""
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(3)
    x, (w, wq, dw) = whole(rng, 60, 48), layer(ops, rng, 33, 48)
    assert not R.Linear8.apply(x, wq, ops, None).requires_grad
    with torch.no_grad():
        assert not R.Linear8.apply(x, wq, ops, dw).requires_grad
    with torch.inference_mode():
        assert torch.equal(R.Linear8.apply(x, wq, ops, dw).double(), x.double() @ w.double().t())
    x.requires_grad_()
    y = R.Linear8.apply(x, wq, ops, None)
    dy = whole(rng, 60, 33)
    y.backward(dy)
    assert torch.equal(x.grad.double(), dy.double() @ w.double()) and not bool(dw.any())


def test_forward_on_a_side_stream(ops):
    """dw, written on the stream of the forward pass, may be read on the caller's stream as soon as backward returns."""
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(10)
    w, wq, dw = layer(ops, rng, 512, 1024)
    x, dy = whole(rng, 2048, 1024), whole(rng, 2048, 512)
    want = dy.double().t() @ x.double()
    side = torch.cuda.Stream()
    for _ in range(5):
        dw.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            y = R.Linear8.apply(x, wq, ops, dw)
        torch.cuda.current_stream().wait_stream(side)
        y.backward(dy)
        assert torch.equal(dw.double(), want)


# ---------------------------------------------------------------------------------------------------- the graph

def test_second_derivatives_are_refused(ops):
    """backward has no graph of its own: differentiating through it raises instead of leaving a part out."""
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(6)
    w, wq, dw = layer(ops, rng, 70, 48)
    x = whole(rng, 60, 48).requires_grad_()
    y = R.Linear8.apply(x, wq, ops, dw)
    g, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        (g.square().sum() + x.square().sum()).backward()


def test_what_is_kept_is_released_and_used_once(ops):
    """After a backward pass the kept activations are freed though y lives on, and a second pass is refused unless the graph was
    retained; retained, it adds to dw again."""
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(7)
    w, wq, dw = layer(ops, rng, 16, 2048)
    x = whole(rng, 4096, 2048)
    dy = whole(rng, 4096, 16)
    y = R.Linear8.apply(x, wq, ops, dw)
    held = torch.cuda.memory_allocated()
    y.backward(dy)
    assert held - torch.cuda.memory_allocated() >= 4096 * 2048            # the 8-bit copy
    once = dw.clone()
    with pytest.raises(RuntimeError):
        y.backward(dy)
    assert torch.equal(dw, once)
    y = R.Linear8.apply(x, wq, ops, dw.zero_())
    y.backward(dy, retain_graph=True)
    y.backward(dy)
    assert torch.equal(dw, 2 * once)


@pytest.mark.parametrize("k", [64, 200])
def test_saved_tensor_hooks_reach_what_is_kept(ops, k):
    """Activations on the host between the passes (rows of 200 bytes come back packed: not a multiple of 16 apart)."""
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(8)
    w, wq, dw = layer(ops, rng, 70, k)
    x = whole(rng, 60, k).requires_grad_()
    dy = whole(rng, 60, 70)
    with torch.autograd.graph.save_on_cpu():
        y = R.Linear8.apply(x, wq, ops, dw)
    y.backward(dy)
    assert torch.equal(x.grad.double(), dy.double() @ w.double()) and torch.equal(dw.double(), dy.double().t() @ x.detach().double())


@pytest.mark.parametrize("k", [48, 200])
def test_weights_changed_between_the_passes_are_noticed(ops, k):
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(9)
    w, wq, dw = layer(ops, rng, 70, k)
    x = whole(rng, 60, k).requires_grad_()
    y = R.Linear8.apply(x, wq, ops, dw)
    wq.scales.mul_(2)
    with pytest.raises(RuntimeError):
        y.backward(torch.ones_like(y))


@pytest.mark.parametrize("k", [48, 200])
def test_weights_made_in_inference_mode(ops, k):
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(11)
    with torch.inference_mode():
        w, wq, _ = layer(ops, rng, 70, k)
    x, dy, dw = whole(rng, 60, k).requires_grad_(), whole(rng, 60, 70), torch.zeros(70, k, device="cuda")
    y = R.Linear8.apply(x, wq, ops, dw)
    y.backward(dy)
    assert torch.equal(x.grad.double(), dy.double() @ w.double()) and torch.equal(dw.double(), dy.double().t() @ x.detach().double())
