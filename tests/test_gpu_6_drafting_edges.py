"""The drafting operators where they once went wrong, and loops of theirs that only larger calls reach: temperatures without end, row starts
out of order, small inputs beside large ones, zero points above 15, tables wider than the workspace, infinities in attended places.
Needs a real MI355X: run with -m gpu."""
import numpy as np
import pytest
import torch

import drafting as D
import test_gpu_4_drafting as T
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


@pytest.mark.parametrize("with_draft", (True, False))
def test_verify_temperature_without_end(with_draft):
    """softmax(logits / T) at T = +inf: the same for every token whose logit is above -inf, and so at 3e38, where the quotients are below
    2^-100.  The definition for these is that of logits which are all 0 or -inf."""
    logits, draft, tokens, u, noise = T.drafts(8, 3, 3001, 61)
    logits[1, :, ::2] = float("-inf")
    draft[2, :, ::3] = float("-inf")
    draft[3, 0, tokens[3, 0].long()] = float("-inf")
    temp = torch.tensor([float("inf")] * 5 + [3e38, 1.0, 0.0])
    print("verify", tuple(logits.shape), temp.tolist(), flush=True)
    out, took, prob = (t.cpu().numpy() for t in B.verify_drafts(logits.cuda(), tokens.cuda(), u.cuda(), noise.cuda(), draft.cuda() if with_draft else None,
                                                                None, temp.cuda()))
    flat = lambda z, t: torch.where(z.isneginf(), z, torch.zeros(())).numpy() if t > 1e38 else z.numpy()  # noqa: E731
    for i in range(8):
        t = float(temp[i])
        want, a, pr, near = D.verify(flat(logits[i], t), tokens[i].numpy(), u[i].numpy(), noise[i].numpy(), flat(draft[i], t) if with_draft else None, 3,
                                     1.0 if t > 1e38 else t)
        assert (abs(prob[i] - pr) <= 2.0 ** -16 * pr).all(), (i, prob[i], pr)
        assert near or (took[i] == a and out[i].tolist() == want), (i, out[i], want)
