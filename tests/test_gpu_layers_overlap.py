"""Products whose result lies in the memory that an operand lies in, on the GPU: refused where they share an element, right where they lie beside one another."""
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


def test_results_over_operands_are_refused(ops):
    import torch
    from paper_2609_23898_b200 import layers
    flat = torch.zeros(8192, device="cuda").bfloat16()
    a, b = flat[:1024].view(16, 64), flat[4096:8192].view(64, 64)
    for out in (flat[8:1032].view(16, 64), flat[1016:2040].view(16, 64), flat[512:1536].view(16, 64), flat[4000:5024].view(16, 64), flat[8191 - 1023:].view(16, 64)):
        before = flat.clone()
        for accumulate in (True, False):
            with pytest.raises(ValueError):
                layers.matmul(ops, a, b, out=out, accumulate=accumulate)
        assert torch.equal(flat, before)
    wide = torch.zeros(16, 128, device="cuda").bfloat16()
    with pytest.raises(ValueError):
        layers.matmul(ops, wide[:, :64], b, out=wide[:, 56:120])
    with pytest.raises(ValueError):
        layers.matmul(ops, b, wide[:, :64], trans_b=True, out=flat[4096:6144].view(64, 32)[:, :16])


@pytest.mark.parametrize("m,k", [(16, 64), (300, 128), (1000, 256)])
def test_results_beside_operands(ops, m, k):
    """Columns of one buffer, and the memory right behind an operand."""
    import torch
    from paper_2609_23898_b200 import layers
    rng = np.random.default_rng(m)

    def whole(*shape):
        return torch.from_numpy(rng.integers(-4, 5, shape).astype(np.float32)).cuda().bfloat16()

    b = whole(k, k)
    wide = whole(m, 2 * k)
    want = wide[:, :k].double() @ b.double()
    layers.matmul(ops, wide[:, :k], b, out=wide[:, k:])
    assert torch.equal(wide[:, k:], want.bfloat16())
    joint = torch.cat((whole(m, k).flatten(), torch.zeros(m * k, device="cuda").bfloat16()))
    want = joint[:m * k].view(m, k).double() @ b.double()
    assert torch.equal(layers.matmul(ops, joint[:m * k].view(m, k), b, out=joint[m * k:].view(m, k)), want.bfloat16())
