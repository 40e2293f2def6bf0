"""The drafting operators where they once went wrong, and loops of theirs that only larger calls reach: temperatures without end, row starts
out of order, small inputs beside large ones, zero points above 15, tables wider than the workspace, infinities in attended places.
Needs a real MI355X: run with -m gpu."""
import numpy as np
import pytest
import torch

import drafting as D
from paper_2501_08090_amd import binding as B

pytestmark = pytest.mark.gpu


def test_append_row_starts_out_of_order_stay_inside_the_table():
    """row starts that do not ascend: what is written is still in pages that the table names.  The rows in front of the table hold a page that
    nobody may reach."""
    c = D.Cache(2, 1, 64, 64)
    before = c.bits()
    cols = 8
    whole = np.full((64 + 4 * cols,), 63, np.int32)
    whole[64:] = np.arange(4 * cols)
    bt = D.dev(whole)[64:].view(4, cols)
    rows = 900
    k = torch.ones((rows, 1, 64), device="cuda")
    cos, sin = torch.ones((rows, 32), device="cuda"), torch.zeros((rows, 32), device="cuda")
    print("append, row starts 0 800 900 0 0", flush=True)
    c.pool.append_rope(0, k, k, cos, sin, bt, D.dev(np.array([0, 800, 900, 0, 0], np.int32)), D.dev(np.zeros(4, np.int32)), index=c.index)
    torch.cuda.synchronize()
    ak, av = c.bits()
    codes, exps = (t.cpu().numpy() for t in c.index.layer_views(0))
    for b in range(cols, 64):  # pages of other requests than the first, which alone has rows in order
        assert np.array_equal(ak[b], before[0][b]) and np.array_equal(av[b], before[1][b]), b
        assert (codes[b] == 0x55).all() and (exps[b] == 0x55).all(), b


def test_append_rows_of_no_request_are_refused():
    c = D.Cache(2, 1, 64, 4)
    k, cs = torch.ones((3, 1, 64), device="cuda"), torch.zeros((3, 32), device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    with pytest.raises(B.ChironError) as e:
        c.pool.append_rope(0, k, k, cs, cs, torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), none, q=k)
    assert e.value.code == -1
    c.pool.append_rope(0, k[:0], k[:0], cs[:0], cs[:0], torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), none)
