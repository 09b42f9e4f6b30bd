"""The workspace of heads' gradient (no GPU): what is made for the largest batch serves every smaller one."""
import ctypes
import random

import pytest

import paper_2310_12670_amd as reft

need = reft.reft_heads_backward_workspace


@pytest.mark.parametrize("cols", [1, 8, 64, 65, 80, 128, 129, 256, 300, 512])
@pytest.mark.parametrize("q,k", [(1, 0), (1, 1), (4, 1), (9, 3), (64, 8), (3, 40), (200, 65), (65535, 65535)])
def test_more_rows_or_heads_need_no_less(q, k, cols):
    rows = sorted({r for n in range(15) for r in (1 << n, (1 << n) + 1, 3 << n, (5 << n) - 1)} | {1000, 2047, 2049, 3000, 4095, 16384, 1 << 20, (1 << 31) - 1})
    sizes = [need(r, q, k, cols) for r in rows]
    assert sizes == sorted(sizes) and 0 < sizes[0] and sizes[-1] <= 512 * 2 * cols * 4
    for r in rows:
        by_heads = [need(r, n, k, cols) for n in (1, 2, 3, 4, 5, 7, 8, 9, 16, 17, 31, 64, 100, 1000)]
        assert by_heads == sorted(by_heads)
        assert all(need(r, q, n, cols) <= need(r, q, n + 1, cols) for n in (0, 1, 2, 3, 7, 8, 15, 63))
        assert need(r, q, k, max(1, cols - 1)) <= need(r, q, k, cols)


def test_calls_take_what_was_made_for_more():
    """Among all sizes of a batch, heads and columns, with keys and without."""
    lib, H, at = reft.binding._load(), reft.binding._Heads, 1 << 20
    rng = random.Random(5)
    for _ in range(3000):
        most = rng.choice([3, 40, 3000, 20000]), rng.choice([1, 9, 64]), rng.choice([1, 8, 80]), rng.choice([16, 80, 128, 512])
        rows, q, k, cols = (rng.randint(1, n) for n in most)
        x, y = ctypes.byref(H(at, 200 * 512, 512)), rng.choice([None, ctypes.byref(H(at, 200 * 512, 512))])
        rc = lib.reft_heads_backward(x, y, x, q, y, k, None, None, None, None, 0, 0, rows, cols, 0, 0, 1e-5, x, y, at, at if y else None, at, need(*most),
                                     reft.binding._CHECK_ONLY)
        assert rc == reft.REFT_OK, (most, rows, q, k, cols)
