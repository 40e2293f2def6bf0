"""How much memory the long-context operators ask for.  No GPU needed."""
import pytest

from paper_2501_08090_amd import binding as B


def workspace(*a):
    return B.load().chiron_row_attention_workspace_bytes(*a)


@pytest.mark.parametrize("heads", ((32, 8, 128), (16, 2, 64), (8, 8, 64), (10, 2, 128), (16, 1, 128)))
@pytest.mark.parametrize("batch,rows", ((64, 64), (1000, 100), (256, 256), (64, 200), (5000, 33), (29, 5000)))
def test_space_goes_by_tiles_not_by_requests(heads, batch, rows):
    """Requests of few rows, or of none, take no part of what the parts of tiles are kept in, whatever max_new promises: 128 columns of d sums, a maximum and
    a divisor for each of at most 16 parts of a tile; beside them 16 columns for each wave of the few rows' kernel and each pass."""
    n_q, n_kv, d = heads
    G = n_q // n_kv
    column, tg = 4 * d + 8, max(1, 16 // G)
    waves = 4 * max(1, 512 // n_kv)
    few = (waves + rows) * n_kv * 16 * column + 16 * rows
    tiles = rows // (128 // G) + min(batch, rows // (tg + 1))
    assert 0 < workspace(n_q, n_kv, d, batch, rows, rows) <= few + tiles * n_kv * 16 * 128 * column + 64


@pytest.mark.parametrize("heads", ((32, 8, 128), (16, 2, 64), (8, 8, 64), (10, 2, 128), (16, 1, 128), (64, 64, 128)))
def test_space_for_the_largest_call_is_enough_for_smaller_ones(heads):
    """a program that takes its workspace once, for the largest batch, rows and max_new that it will bring"""
    sizes = (1, 2, 3, 4, 5, 8, 16, 17, 29, 33, 64, 100, 129, 500, 512, 1023, 1501, 2048, 4096, 5003, 16384)
    space = {(b, r, m): workspace(*heads, b, r, m) for b in sizes for r in sizes for m in sizes}
    for (b, r, m), n in space.items():
        for i in range(3):  # one of them a size smaller, and so on down
            at = sizes.index((b, r, m)[i])
            if at:
                less = [b, r, m]
                less[i] = sizes[at - 1]
                assert space[tuple(less)] <= n, (less, (b, r, m))
    assert workspace(32, 8, 128, 4, 16384, 16384) >= max(workspace(32, 8, 128, 4, r, r) for r in range(1, 3000))
