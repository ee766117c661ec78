"""The embedding gradient's sort by digits, on the GPU: one to four digits, lists on both sides of where it begins, tiles above the usual size, the longest pieces.

Tolerance: n additions in binary32 within n 2^-24 of the sum of magnitudes, the scale's product, the addition to what is there (two roundings more each).
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ops():
    import torch
    from paper_2609_23898_b200 import training
    assert torch.cuda.is_available()
    o = training.Ops()
    yield o
    o.status()


def digits(vocab):
    """Digits of up to 9 bits of the largest key (vocab itself: padding)."""
    return -(-vocab.bit_length() // 9)


def ids_of(kind, tokens, vocab):
    import torch
    rng = np.random.default_rng(tokens)
    if kind == "zipf":
        i = np.minimum(np.exp(rng.random(tokens) * np.log(vocab + 1)).astype(np.int64) - 1, vocab - 1)
    elif kind == "one":
        i = np.full(tokens, vocab - 1)
    elif kind == "padded":
        i = rng.integers(-vocab, vocab, tokens)
    else:
        i = rng.integers(0, vocab, tokens)
    i[:3] = vocab - 1, 0, vocab - 1
    return torch.from_numpy(i.astype(np.int64)).cuda()


def check(ops, ids, vocab, width, accumulate):
    import torch
    from paper_2609_23898_b200 import layers
    tokens = ids.numel()
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    dy = torch.randn(tokens, width, device="cuda", generator=g)
    d = torch.full((vocab, width), 2.0, device="cuda")
    layers.embed_backward(ops, dy, ids, d, scale=0.75, accumulate=accumulate)
    live = ids >= 0
    flat, start = ids[live], 2.0 if accumulate else 0.0
    # only rows that some token names are compared value by value: of a large table nearly all have none
    named, place = flat.unique(return_inverse=True)
    want, size = (torch.zeros(named.numel(), width, dtype=torch.float64, device="cuda").index_add_(0, place, v) for v in (dy[live].double(), dy[live].double().abs()))
    n = torch.bincount(place)[:, None]
    off = (d[named].double() - (0.75 * want + start)).abs()
    assert bool((off <= (0.75 * size + start) * (n + 4) * U).all()), float(off.max())
    d[named] = start
    assert bool((d == start).all())


@pytest.mark.parametrize("accumulate", [True, False])
@pytest.mark.parametrize("kind", ["uniform", "zipf", "padded", "one"])
@pytest.mark.parametrize("vocab", [300, (1 << 9) - 1, 1 << 9, (1 << 18) - 1, 1 << 18, (1 << 18) + 1, (1 << 27) - 1, (1 << 27) + 5])
def test_digits(ops, vocab, kind, accumulate):
    from paper_2609_23898_b200 import cerar
    assert cerar.lib.cerar_embed_grad_workspace(9000, vocab, 2) >= 16 * 9000           # two lists of keys and numbers: this length is sorted by digits
    check(ops, ids_of(kind, 9000, vocab), vocab, 2, accumulate)


def test_all_numbers_of_digits_are_tested():
    vocabs = [m.args[1] for m in test_digits.pytestmark if m.name == "parametrize" and m.args[0] == "vocab"][0]
    assert {digits(v) for v in vocabs} == {1, 2, 3, 4}


@pytest.mark.parametrize("accumulate", [True, False])
@pytest.mark.parametrize("kind", ["uniform", "zipf", "padded", "one"])
@pytest.mark.parametrize("tokens,vocab,width", [(8192, 1000, 3), (8193, 1000, 3), (32769, 5000, 2), (131072, 70000, 2), (131073, 70000, 2), (140001, 400, 2), (524288, 600, 1),
                                                (524289, 600, 1), (600011, 70000, 1), (600011, 300000, 2), (1100003, 1000, 1)])
def test_lengths(ops, tokens, vocab, width, kind, accumulate):
    """Where the sort by digits begins (8193 tokens), where pieces become longer (32,769 and 131,073), where tiles do (524,289)."""
    check(ops, ids_of(kind, tokens, vocab), vocab, width, accumulate)


def test_the_order_of_equal_tokens_is_kept(ops):
    """Four values to a row, of magnitudes so far apart that their order shows in the sum: equal bits, over three digits."""
    import torch
    from paper_2609_23898_b200 import layers
    vocab, tokens = 300000, 8 * 1500
    rows = torch.randperm(vocab, device="cuda")[:tokens // 4]
    ids = rows.repeat(4)[torch.randperm(tokens, device="cuda")]
    dy = torch.randn(tokens, 1, device="cuda").double().mul(20).exp2().float()         # magnitudes from 2^-80 to 2^80
    d = torch.zeros(vocab, 1, device="cuda")
    layers.embed_backward(ops, dy, ids, d, accumulate=False)
    # the four lie next to one another in the sorted list, and no piece (16 tokens here) ends between them
    order = torch.sort(ids, stable=True).indices.view(-1, 4)
    v = dy[order, 0]
    want = ((v[:, 0] + v[:, 1]) + v[:, 2]) + v[:, 3]
    assert torch.equal(d[ids[order[:, 0]], 0], want)
