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
