"""kv_tables_grow (include/kvr_tables.h) where the list of free blocks holds ids that are
no block."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_tables import Call, loop, request_set  # noqa: E402


@pytest.mark.gpu
@pytest.mark.parametrize("R,low,high,grow,B", [(1, 40, 40, 0, 16), (64, 20, 90, 3, 16), (300, 0, 200, 0, 24), (9, 0, 30, 4, 1)])
def test_negative_ids_in_the_free_list(R, low, high, grow, B):
    """They are handed out like the others; their rows have no slot, but count as placed."""
    held, lens, free, tables = request_set(R, low, high, grow, B, seed=R)
    free = free[:max(1, int((lens - held).sum()) // B)].copy()
    free[::3] = -1000 - np.arange(len(free[::3]))
    total = int((lens - held).sum())
    c = Call(held, lens, B, free, tables, total + 7)
    c.run()
    tables, offsets, slots, positions, counts = loop(held, lens, B, free, tables, total + 7)
    counts[3] -= sum(tables[r, p // B] <= -1000 for r in range(R) for p in range(held[r], lens[r]))
    c.check((tables, offsets, slots, positions, counts))
