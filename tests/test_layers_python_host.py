"""layers.py's own decisions, without a device."""
import random


def test_meeting_matrices():
    """Against the sets of their bytes."""
    from paper_2609_23898_b200 import layers
    rng = random.Random(1)
    seen = {True: 0, False: 0}
    for i in range(20000):
        sizes = []
        for _ in range(2):
            width = rng.randint(0, 6)
            sizes.append([rng.randint(0, 60), rng.randint(0, 6), width, width + rng.randint(0, 8) + (width == 0)])
        sizes[1][2:] = [2 * ((v + 1) // 2) for v in sizes[1][2:]]             # (bfloat16)
        if i % 2:
            sizes[0][3] = sizes[1][3] = max(sizes[0][3], sizes[1][3], sizes[0][2], sizes[1][2]) // 2 * 2 + 2
        held = [{p + r * pitch + e for r in range(rows) for e in range(width)} for p, rows, width, pitch in sizes]
        want = bool(held[0] & held[1])
        assert layers._meet(*sizes[0], *sizes[1][:2], sizes[1][2] // 2, sizes[1][3] // 2) == want, sizes
        seen[want] += 1
    assert min(seen.values()) > 4000


def test_nothing_is_kept_where_no_backward_pass_can_follow(monkeypatch):
    """Gated keeps g and u where x or a weight gradient will be wanted of it, and never under no_grad or in inference mode."""
    import torch
    from paper_2609_23898_b200 import layers
    kept = []

    def gated(ops, x, w_in, w_out, *, activation="silu", keep=False):
        kept.append(keep)
        y = x.new_zeros(*x.shape[:-1], w_out.size(0))
        return (y, (x, x.new_zeros(8, dtype=torch.uint8), activation)) if keep else y

    monkeypatch.setattr(layers, "gated", gated)
    w_in, w_out, dw = torch.zeros(6, 4).bfloat16(), torch.zeros(4, 3).bfloat16(), torch.zeros(6, 4)
    for follows in (False, True):
        for wanted in (None, dw):
            x = torch.zeros(5, 4).bfloat16().requires_grad_(follows)
            y = layers.Gated.apply(x, w_in, w_out, None, wanted, None)
            assert kept.pop() == (follows or wanted is not None) == y.requires_grad
            for mode in (torch.no_grad, torch.inference_mode):
                with mode():
                    y = layers.Gated.apply(x, w_in, w_out, None, wanted, None)
                    assert kept.pop() is False and not y.requires_grad
    assert not kept
