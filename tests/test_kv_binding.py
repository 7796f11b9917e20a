"""The 4-bit cache's binding on the host: no call here reaches a kernel."""
import random

import paper_2608_03839_amd as oil


def test_kept_workspaces_are_bounded():
    """Buffers of a stream, whatever sizes its calls had and in whatever order."""
    rng = random.Random(1)
    for order in ("random", "up", "down"):
        needs = [rng.randrange(1, 1 << 20) for _ in range(500)]
        needs = needs if order == "random" else sorted(needs, reverse=order == "down")
        kept = oil._Workspaces()
        for i, n in enumerate(needs):
            ws = kept.get(("attend", (i,)), n, "cpu")
            assert ws.numel() == n and kept.by_sizes["attend", (i,)] is ws
            held = [b.data_ptr() for b in kept.buffers]
            assert ws.data_ptr() in held      # whoever holds an address has its buffer kept
        assert sum(b.numel() for b in kept.buffers) <= 4 * max(needs)


def test_remembered_sizes_are_bounded():
    kept = oil._Workspaces()
    for i in range(2 * kept.SIZES + 5):
        kept.get(("evict", (i, 1)), 64, "cpu")
    assert len(kept.by_sizes) <= kept.SIZES and len(kept.buffers) == 1
