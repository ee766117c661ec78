"""The products of the gated block's gradient beside one another on the GPU: results do not depend on which of them are wanted, on what runs in front, or on
dx lying over dy.  Equal bits, no tolerance."""
import ctypes as C

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


def weights(t, d, f, o, seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + t + d + f)

    def normal(*s, std=1.0):
        return (torch.randn(*s, device="cuda", generator=g) * std).bfloat16()

    return normal(t, d), normal(2 * f, d, std=1.5 * d ** -0.5), normal(o, f, std=f ** -0.5), normal(t, o)


# one turn of tiles; dw_out in several; dx and dw_in in several; rows that are copied to other boundaries
SIZES = [(64, 256, 512, 256), (200, 2304, 2312, 2304), (3000, 2048, 520, 2048), (333, 520, 1377, 520), (9, 40, 24, 40)]


@pytest.mark.parametrize("t,d,f,o", SIZES)
def test_dx_over_dy(ops, t, d, f, o):
    import torch
    from paper_2609_23898_b200 import cerar, layers
    cases = [weights(t, d, f, o, s) for s in range(8)]
    runs = []
    for x, w_in, w_out, dy in cases:
        _, kept = layers.gated(ops, x, w_in, w_out, keep=True)
        dw = [torch.zeros_like(w_in), torch.zeros_like(w_out)]
        dx = layers.gated_backward(ops, dy, kept, w_in, w_out, *dw)
        torch.cuda.synchronize()
        over, got = dy.clone(), [torch.zeros_like(w_in), torch.zeros_like(w_out)]
        b = cerar.GatedBlock(tokens=t, width=d, hidden=f, outputs=o, activation=0, accumulate=0, x=kept[0].data_ptr(), ldx=d, w_in=w_in.data_ptr(), ldw_in=d, w_out=w_out.data_ptr(),
                             ldw_out=f, kept=kept[1].data_ptr(), dy=over.data_ptr(), lddy=o, dx=over.data_ptr(), lddx=d, dw_in=got[0].data_ptr(), lddw_in=d, dw_in_type=1,
                             dw_out=got[1].data_ptr(), lddw_out=f, dw_out_type=1)
        ws = torch.empty(cerar.lib.cerar_gated_workspace(C.addressof(b), 1), dtype=torch.uint8, device="cuda")
        runs.append((kept, b, ws, over, got, dx, dw))
    torch.cuda.synchronize()
    for _, b, ws, *_ in runs:
        assert cerar.lib.cerar_gated_backward(ops._h, C.addressof(b), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    for _, _, _, over, got, dx, dw in runs:
        assert torch.equal(over, dx) and torch.equal(got[0], dw[0]) and torch.equal(got[1], dw[1])
    ops.status()


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("wanted", [(1, 1, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)])
@pytest.mark.parametrize("t,d,f,o", SIZES)
def test_every_choice_of_results_without_a_pause(ops, t, d, f, o, wanted, captured):
    """Passes one behind the other in the same memory, with some of dw_out, dx and dw_in wanted: the bits of a pass alone with all of them."""
    import torch
    from paper_2609_23898_b200 import layers
    cases = [weights(t, d, f, o, s) for s in range(6)]

    def run(case, wanted):
        x, w_in, w_out, dy = case
        _, kept = layers.gated(ops, x, w_in, w_out, keep=True)
        dw_in, dw_out = (torch.ones_like(w, dtype=torch.float32) if want else None for w, want in ((w_in, wanted[2]), (w_out, wanted[0])))
        return dw_out, layers.gated_backward(ops, dy, kept, w_in, w_out, dw_in, dw_out, need_dx=bool(wanted[1])), dw_in

    want = []
    for case in cases:
        want.append(run(case, (1, 1, 1)))
        torch.cuda.synchronize()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = [run(case, wanted) for case in cases]
        for _ in range(2):
            graph.replay()
    else:
        got = [run(case, wanted) for case in cases]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        for p, q, w in zip(a, b, wanted):
            assert (p is None) == (not w) and (p is None or torch.equal(p, q))
    ops.status()


def test_one_and_several_turns_are_tested():
    """Of every product's tiles, on 148 SMs."""
    from paper_2609_23898_b200 import cerar

    def turns(m, n, k):
        split = C.c_int()
        form = cerar.lib.cerar_matmul_bf16_tile(m, n, k, 148, C.byref(split))
        rows, cols, blocks = ((256, 256, 2), (256, 128, 2), (128, 128, 1))[form]
        return -(-m // rows) * -(-n // cols) * split.value * blocks > 148

    for product in (lambda t, d, f, o: (o, f, t), lambda t, d, f, o: (t, d, 2 * f), lambda t, d, f, o: (2 * f, d, t)):
        assert {turns(*product(*s)) for s in SIZES} == {True, False}
