"""The drafting operators together: a draft step with lossless 4-bit weights and all pages against the decode step, greedy draft and
verify against plain greedy decoding, and the example as it is run.  Needs a real MI355X: run with -m gpu."""
import numpy as np
import pytest
import torch

from paper_2501_08090_amd import binding as B
from paper_2501_08090_amd import drafting as DV
from paper_2501_08090_amd import inputs as I

pytestmark = pytest.mark.gpu


def lossless(shape, g, group):
    """bf16 weights that quantize4 keeps exactly: whole multiples, -7 .. 7, of 2^-8, 7 among every group's"""
    q = torch.randint(-7, 8, shape, generator=g)
    q[:, ::group] = 7
    return (q * 2.0 ** -8).to(torch.bfloat16).cuda()


def setup(m, lens, room, weights, group, top, max_rows, seed=0):
    bt, blocks = I.make_block_table(lens + room, seed=seed)
    model = B.Model(m, max_rows, bt.shape[1])
    model.load_weights(weights)
    mem = torch.empty(blocks * model.kv_block_bytes(), dtype=torch.uint8, device="cuda")
    mem.view(torch.int16).fill_(0x7FC0)
    pool = B.KVPool(model, memory=mem)
    btd = torch.from_numpy(bt).cuda()
    si, ps = I.prefill_index(lens)
    for l in range(m["n_layers"]):
        k, v = I.make_kv_layer(m, len(si), l, seed=seed, device="cuda")
        pool.append(l, k, v, btd, torch.from_numpy(si).cuda(), torch.from_numpy(ps).cuda())
    d = DV.Drafter(model, pool, weights, group=group, top=top)
    sl = torch.from_numpy(lens).cuda()
    d.index.update(btd, torch.zeros_like(sl), sl, int(lens.max()))
    return d, btd, sl


@pytest.mark.parametrize("group", (32, 64, 128))
def test_draft_step_is_the_decode_step_with_lossless_weights_and_all_pages(group):
    """tolerance: two implementations of one decoder, 1e-3 of the logits' deviation (the whole-step tests allow 2e-2)"""
    m = dict(I.TINY, ffn=384, vocab=1000)
    g = torch.Generator().manual_seed(1)
    H, F = m["hidden"], m["ffn"]
    shapes = I.matrix_shapes(m)
    w = {n: [lossless(shapes[n], g, group) for _ in range(2)] for n in I.LAYER_MATRICES}
    w["embed"] = torch.randn((m["vocab"], H), generator=g).to(torch.bfloat16).cuda()
    w["lm_head"] = lossless((m["vocab"], H), g, group)
    for n in ("attn_norm", "ffn_norm"):
        w[n] = [(1 + 0.1 * torch.randn(H, generator=g)).to(torch.bfloat16).cuda() for _ in range(2)]
    w["final_norm"] = (1 + 0.1 * torch.randn(H, generator=g)).to(torch.bfloat16).cuda()
    lens = np.array([5, 63, 64, 200, 0], np.int32)
    d, bt, sl = setup(m, lens, 8, w, group, 64, 16)
    tokens = torch.tensor([1, 2, 3, 999, 0], dtype=torch.int32, device="cuda")
    got = d.step(bt, sl, tokens)
    k, v = (t.clone() for t in d.pool.layer_views(1))
    want = B.decode_step(d.model, d.pool, bt, sl, tokens)
    assert (got - want).abs().max().item() <= 1e-3 * want.std().item()
    k2, v2 = d.pool.layer_views(1)
    near = lambda a, b: ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 1e-3).logical_or(b.isnan() & a.isnan()).all()  # noqa: E731
    assert near(k, k2) and near(v, v2)  # the step has written the same slots


@pytest.mark.parametrize("drafts,top", ((1, 4), (3, 4), (5, 64)))
def test_greedy_rounds_are_greedy_decoding(drafts, top):
    m = dict(I.TINY)
    w = I.make_weights(m, seed=3, device="cuda", std=0.05)
    lens = np.array([100, 7, 300], np.int32)
    new = 14
    d, bt, sl = setup(m, lens, 40, w, 64, top, 24, seed=3)
    first = torch.tensor([11, 12, 13], dtype=torch.int32, device="cuda")
    # plain greedy decoding on a pool of its own
    p, _, pl = setup(m, lens, 40, w, 64, top, 24, seed=3)
    want, t, s = [], first, pl.clone()
    for _ in range(new):
        t = B.decode_step(p.model, p.pool, bt, s, t).argmax(-1).to(torch.int32)
        s = s + 1
        want.append(t.tolist())
    want = np.array(want).T
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    got, tokens, taken = [[] for _ in lens], first, 0
    zero = torch.zeros(3, device="cuda")
    while min(len(x) for x in got) < new:
        out, accepted, sl, tokens = DV.draft_and_verify(d, bt, sl, tokens, drafts, zero, g)
        taken += int(accepted.sum())
        for i, row in enumerate(out.tolist()):
            n = int(accepted[i])
            assert all(x >= 0 for x in row[:n + 1]) and row[n + 1:] == [-1] * (drafts - n)
            got[i] += row[:n + 1]
        assert sl.tolist() == [int(lens[i]) + len(got[i]) for i in range(3)]
        if max(len(x) for x in got) > 35:
            break
    print("accepted", taken, flush=True)
    for i in range(3):
        n = min(new, len(got[i]))
        assert got[i][:n] == want[i, :n].tolist(), i


def test_sampled_rounds_keep_the_index_and_the_lengths():
    m = dict(I.TINY)
    w = I.make_weights(m, seed=5, device="cuda", std=0.02)
    lens = np.array([31, 16, 250, 1], np.int32)
    d, bt, sl = setup(m, lens, 60, w, 32, 6, 24, seed=5)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    tokens = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device="cuda")
    temp = torch.tensor([0.5, 1.0, 0.0, 2.0], device="cuda")
    for _ in range(6):
        before = sl.clone()
        out, accepted, sl, tokens = DV.draft_and_verify(d, bt, sl, tokens, 4, temp, g)
        assert torch.equal(sl, before + accepted + 1)
        assert ((out >= 0).sum(1) == accepted + 1).all() and (out < m["vocab"]).all()
    # the index kept on the way is the index made afresh (records of the pages that hold tokens of the model alone)
    kept = [t.clone() for t in d.index.layer_views(1)]
    d.index.update(bt, torch.zeros_like(sl), sl, 512)
    fresh = d.index.layer_views(1)
    for i in range(4):
        pages = bt[i, :-(-int(sl[i]) // 16)].long()
        assert torch.equal(kept[0][pages], fresh[0][pages]) and torch.equal(kept[1][pages], fresh[1][pages])


def test_example_runs(capsys):
    DV.main(["--steps", "2", "--drafts", "3", "--batch", "2", "--context", "100", "--top", "4"])
    assert "drafted tokens accepted" in capsys.readouterr().out
