"""The drafting operators on the GPU against their definitions in 64 bits: rotate-and-append with the page index, page selection,
attention over listed pages, verification of drafts, 4-bit products.  Needs a real MI355X: run with -m gpu.

Tolerances.  Whole numbers (index records, page lists, tokens) are equal.  Stored bf16 keys: half a unit in the last place of the
exact value plus the fp32 rounding of two products.  Attention: a softmax whose logits are off by at most s moves an average of
values by at most 2 s max|v|, with s from the products' own magnitudes, plus 2^-20 max|v| for the exponentials and the sums.
Probabilities: 2^-16 relative (logits up to 100 in an fp32 exponential).  4-bit products: 2^-23 of the largest |x| of its 128 inputs per
product, and the fp32 additions over the groups."""
import numpy as np
import pytest
import torch

import drafting as D
from paper_2501_08090_amd import binding as B

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


# ---- rotate and append ---------------------------------------------------------------------------------------------

def append_case(n_q, n_kv, d, old, new, dtype, seed, layer=0, layers=1, shift=0, contiguous=False, with_q=True, with_index=True):
    rng = np.random.default_rng(seed)
    total = [a + b for a, b in zip(old, new)]
    bt, blocks = D.tables(total, seed)
    c = D.Cache(n_q, n_kv, d, blocks, layers=layers, index=with_index)
    bt = D.widen(bt, bt.shape[1] + 2)
    # the old tokens, through the plain append
    si = np.repeat(np.arange(len(old)), old).astype(np.int32)
    ps = np.concatenate([np.arange(n) for n in old] + [np.zeros(0)]).astype(np.int32)
    btd = D.dev(bt)
    if len(si):
        kv = torch.from_numpy(rng.standard_normal((2, len(si), n_kv, d))).to(torch.bfloat16).cuda()
        c.pool.append(layer, kv[0].contiguous(), kv[1].contiguous(), btd, D.dev(si), D.dev(ps))
    before = c.bits(layer)
    rows = sum(new)
    width = (n_q + 2 * n_kv) * d + (0 if contiguous else 64) + shift
    fused = torch.from_numpy(rng.standard_normal((rows, width))).to(dtype).cuda()
    q = fused[:, shift:shift + n_q * d].unflatten(1, (n_q, d))
    k = fused[:, shift + n_q * d:shift + (n_q + n_kv) * d].unflatten(1, (n_kv, d))
    v = fused[:, shift + (n_q + n_kv) * d:shift + (n_q + 2 * n_kv) * d].unflatten(1, (n_kv, d))
    if contiguous:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    pos = np.concatenate([np.arange(a, a + b) for a, b in zip(old, new)]).astype(np.int32)
    cos, sin = B.rope_table(D.dev(pos), d, 10000.0)
    say("append", n_q, n_kv, d, dtype, "old", old, "new", new, "shift", shift)
    got = c.pool.append_rope(layer, k, v, cos, sin, btd, D.dev(starts), D.dev(np.array(old, np.int32)), q=q if with_q else None, index=c.index)
    torch.cuda.synchronize()
    return c, bt, before, fused, q, k, v, cos.cpu().numpy(), sin.cpu().numpy(), starts, pos, got


def check_append(n_q, n_kv, d, old, new, dtype, seed, layer=0, **kw):
    c, bt, before, fused, q, k, v, cos, sin, starts, pos, got = append_case(n_q, n_kv, d, old, new, dtype, seed, layer=layer, **kw)
    kd, vd, qd = (t.double().cpu().numpy() for t in (k, v, q))
    ang = pos[:, None] * 10000.0 ** (-2.0 * np.arange(d // 2) / d)
    assert abs(cos - np.cos(ang)).max() < 1e-7 and abs(sin - np.sin(ang)).max() < 1e-7
    want_q, want_k = D.rotate(qd, cos, sin), D.rotate(kd, cos, sin)
    if got is not None:
        big = abs(qd).reshape(len(pos), n_q, 2, d // 2).sum(2)
        assert (abs(got.double().cpu().numpy() - want_q) <= np.concatenate((big, big), -1) * 2.0 ** -22).all()
    else:
        assert kw.get("with_q") is False
    after_k, after_v = c.bits(layer)
    keys, values = c.keys(layer), c.values(layer)
    touched = np.zeros(after_k.shape[:2], bool)
    vr = v.to(torch.bfloat16).double().cpu().numpy()
    for i in range(len(old)):
        for j in range(new[i]):
            r, p = starts[i] + j, old[i] + j
            b, s = bt[i, p // 16], p % 16
            touched[b, s] = True
            big = abs(kd[r]).reshape(n_kv, 2, d // 2).sum(1)
            half = np.ldexp(1.0, np.frexp(want_k[r])[1] - 9)  # half a unit in the last of 8 significant bits
            tol = half + np.concatenate((big, big), -1) * 2.0 ** -22
            assert (abs(keys[b, s] - want_k[r]) <= tol).all(), (i, j)
            assert np.array_equal(values[b, s], vr[r]), (i, j)
    assert np.array_equal(after_k[~touched], before[0][~touched]) and np.array_equal(after_v[~touched], before[1][~touched])
    if c.index is not None:
        codes, exps = (t.cpu().numpy() for t in c.index.layer_views(layer))
        seen = set()
        for i in range(len(old)):
            for pg in range(old[i] // 16, -(-(old[i] + new[i]) // 16) if new[i] else 0):
                n = min(16, old[i] + new[i] - pg * 16)
                for h in range(n_kv):
                    want, e = D.record(keys[bt[i, pg], :n, h])
                    assert exps[bt[i, pg], h] == e and np.array_equal(codes[bt[i, pg], h], want), (i, pg, h)
                seen.add(int(bt[i, pg]))
        rest = [b for b in range(c.blocks) if b not in seen]
        assert (codes[rest] == 0x55).all() and (exps[rest] == 0x55).all()


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("shift", (0, 1))
def test_append_more_queries_than_the_caches_hold(dtype, shift):
    check_append(16, 1, 128, old=[0, 7], new=[2200, 2000], dtype=dtype, seed=21, shift=shift)


@pytest.mark.parametrize("requests", (63, 64, 65, 150))
def test_append_many_requests(requests):
    check_append(4, 2, 64, old=[i * 11 % 40 for i in range(requests)], new=[i * 7 % 5 for i in range(requests)], dtype=torch.bfloat16, seed=22)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("heads", ((4, 2, 64), (8, 8, 128), (16, 1, 128), (12, 12, 64)))
def test_append_rope_ragged(heads, dtype):
    check_append(*heads, old=[0, 15, 16, 5, 40, 31], new=[1, 1, 1, 0, 37, 18], dtype=dtype, seed=3)


@pytest.mark.parametrize("old,new", (([0], [1]), ([7], [3]), ([3], [13]), ([3], [14]), ([0], [100]), ([1], [255]), ([0, 0, 0], [0, 2, 0]), ([17] * 9, [1] * 9)))
def test_append_rope_page_borders(old, new):
    check_append(4, 2, 128, old, new, torch.float32, 5)


@pytest.mark.parametrize("shift", (1, 2, 3, 4))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_append_rope_rows_that_are_not_aligned(shift, dtype):
    check_append(4, 2, 64, [9, 0], [20, 7], dtype, 11, shift=shift)


def test_append_rope_contiguous_without_queries_or_index_in_a_later_layer():
    check_append(4, 2, 64, [9, 0, 30], [20, 7, 1], torch.bfloat16, 12, layer=2, layers=3, contiguous=True)
    check_append(4, 2, 64, [9, 0, 30], [20, 7, 1], torch.float32, 13, layer=1, layers=3, with_q=False, with_index=False)


def test_append_rope_many_requests():
    rng = np.random.default_rng(8)
    check_append(2, 1, 64, rng.integers(0, 60, 150).tolist(), rng.integers(0, 40, 150).tolist(), torch.float32, 8)


def test_append_rope_skips_pages_that_are_none():
    """a page id of -1 or behind the pool, and positions behind the table, write nothing"""
    c = D.Cache(2, 1, 64, 4)
    before = c.bits()
    bt = np.array([[-1, 4, 2]], np.int32)
    rows = 60  # 4 pages: none, behind the pool, page 2, behind the table
    k = torch.ones((rows, 1, 64), device="cuda")
    cos, sin = torch.ones((rows, 32), device="cuda"), torch.zeros((rows, 32), device="cuda")
    c.pool.append_rope(0, k, k, cos, sin, D.dev(bt), D.dev(np.array([0, rows], np.int32)), D.dev(np.array([0], np.int32)), index=c.index)
    torch.cuda.synchronize()
    ak, av = c.bits()
    assert (ak[2] == 0x3F80).all() and (av[2] == 0x3F80).all()
    for b in (0, 1, 3):
        assert np.array_equal(ak[b], before[0][b]) and np.array_equal(av[b], before[1][b])
    codes, exps = (t.cpu().numpy() for t in c.index.layer_views(0))
    assert (codes[2] == 64).all() and (exps[2] == -6).all() and (codes[[0, 1, 3]] == 0x55).all()


def special_keys(rng, n, n_kv, d):
    k = torch.from_numpy(rng.standard_normal((n, n_kv, d))).to(torch.bfloat16)
    flat = k.view(-1)
    pick = rng.permutation(flat.numel())[:24]
    for at, val in zip(pick, [float("nan"), float("inf"), float("-inf"), 3.3e38, -3.3e38, 1e-39, -1e-39, 0.0] * 3):
        flat[at] = val
    return k


@pytest.mark.parametrize("d", (64, 128))
def test_index_update_and_keys_of_every_kind(d):
    rng = np.random.default_rng(d)
    lens = [1, 16, 17, 50, 0, 33]
    bt, blocks = D.tables(lens, 4)
    c = D.Cache(2, 2, d, blocks, layers=2)
    si, ps = np.repeat(np.arange(6), lens).astype(np.int32), np.concatenate([np.arange(n) for n in lens]).astype(np.int32)
    n = len(si)
    k = special_keys(rng, n, 2, d)
    k[0] = 0                                   # all keys 0: exponent 0
    k[1:17, 0] = 1e-39                         # denormal keys
    k[17:34, 1] = 127.0 * 2.0 ** -9            # exactly 127 steps
    k[34:84, 0, :] = 255.0 * 2.0 ** 3          # between 127 and 128 of the smaller power
    for layer in range(2):
        c.pool.append(layer, k.cuda(), k.cuda(), D.dev(bt), D.dev(si), D.dev(ps))
    first = np.array([0, 0, 16, 20, 0, 32], np.int32)
    say("index update", d)
    c.index.update(D.dev(bt), D.dev(first), D.dev(np.array(lens, np.int32)), max_new=64, layer=1, n_layers=1)
    torch.cuda.synchronize()
    keys = c.keys(1)
    codes, exps = (t.cpu().numpy() for t in c.index.layer_views(1))
    seen = set()
    for i, L in enumerate(lens):
        for pg in range(first[i] // 16, -(-L // 16)):
            for h in range(2):
                want, e = D.record(keys[bt[i, pg], :min(16, L - pg * 16), h])
                assert exps[bt[i, pg], h] == e and np.array_equal(codes[bt[i, pg], h], want), (i, pg, h)
            seen.add(int(bt[i, pg]))
    rest = [b for b in range(c.blocks) if b not in seen]
    assert (codes[rest] == 0x55).all()
    assert (c.index.layer_views(0)[0] == 0x55).all()
    # both layers, and no more pages than max_new says: request 3 stops after the pages of 1 + 14 positions
    c.index.update(D.dev(bt), D.dev(np.zeros(6, np.int32)), D.dev(np.array(lens, np.int32)), max_new=2)
    torch.cuda.synchronize()
    codes0 = c.index.layer_views(0)[0].cpu().numpy()
    assert np.array_equal(codes0[bt[3, 0], 0], D.record(c.keys(0)[bt[3, 0], :16, 0])[0])
    assert (codes0[bt[3, 2]] == 0x55).all() and (codes0[bt[3, 3]] == 0x55).all()


# ---- selection -----------------------------------------------------------------------------------------------------

def filled(n_q, n_kv, d, lens, seed, max_batch=64, cols=None, spread=True, layers=1, layer=0, pages=None):
    rng = np.random.default_rng(seed)
    bt, blocks = D.tables(lens, seed)
    if pages is not None:
        bt, blocks = pages
    bt = D.widen(bt, cols or bt.shape[1])
    c = D.Cache(n_q, n_kv, d, blocks, max_batch=max_batch, max_blocks=bt.shape[1], layers=layers)
    si, ps = np.repeat(np.arange(len(lens)), lens).astype(np.int32), np.concatenate([np.arange(n) for n in lens]).astype(np.int32)
    if len(si):
        k = rng.standard_normal((len(si), n_kv, d)) * (2.0 ** rng.integers(-3, 3, (len(si), 1, 1)) if spread else 1.0)
        v = rng.standard_normal((len(si), n_kv, d))
        k, v = (torch.from_numpy(t).to(torch.bfloat16).cuda() for t in (k, v))
        c.pool.append(layer, k, v, D.dev(bt), D.dev(si), D.dev(ps))
        c.index.update(D.dev(bt), D.dev(np.zeros(len(lens), np.int32)), D.dev(np.array(lens, np.int32)), max(lens), layer=layer, n_layers=1)
    return c, bt


def check_select(c, bt, q, ctx, seq, top, n_first, n_last, layer=0, pass_seq=True):
    say("select", c.n_q, c.n_kv, c.d, "rows", len(ctx), "top", top, n_first, n_last, "longest", max(ctx))
    pages, counts = B.op_select_pages(c.model, c.pool, c.index, layer, q, D.dev(bt), D.dev(np.array(ctx, np.int32)), top, n_first=n_first,
                                      n_last=n_last, row_seq=D.dev(np.array(seq, np.int32)) if pass_seq else None)
    got, cnt = pages.cpu().numpy(), counts.cpu().numpy()
    codes, exps = (t.cpu().numpy().astype(np.int64) for t in c.index.layer_views(layer))
    qn = q.double().cpu().numpy().reshape(len(ctx), c.n_kv, c.G, c.d)
    for r in range(len(ctx)):
        n = -(-max(ctx[r], 0) // 16)
        assert cnt[r] == min(n, top)
        blocks = bt[seq[r], :n]
        for h in range(c.n_kv):
            want = D.select(qn[r, h], codes[blocks, h], exps[blocks, h], ctx[r], top, n_first, n_last)
            assert got[r, h].tolist() == want + [-1] * (top - len(want)), (r, h)
    return pages, counts


@pytest.mark.parametrize("heads", ((1, 1, 64), (4, 2, 64), (8, 2, 128), (8, 1, 128), (16, 1, 64), (32, 2, 128), (4, 4, 128)))
def test_select_pages_head_layouts(heads):
    lens = [400, 1, 0, 16, 17, 333, 95]
    c, bt = filled(*heads, lens, 21)
    q = torch.randn((7, heads[0] * heads[2]), generator=torch.Generator().manual_seed(1)).cuda()
    check_select(c, bt, q, lens, range(7), 5, 1, 1, pass_seq=False)


@pytest.mark.parametrize("top,n_first,n_last", ((1, 0, 0), (1, 1, 0), (1, 0, 1), (2, 1, 1), (7, 3, 4), (16, 0, 2), (40, 1, 1), (41, 1, 1), (64, 2, 2)))
def test_select_pages_counts_and_forced_pages(top, n_first, n_last):
    c, bt = filled(4, 1, 64, [650, 640, 641, 100], 22)
    ctx, seq = [650, 640, 641, 100, 649, 1, 0, 16], [0, 1, 2, 3, 0, 0, 0, 2]
    q = torch.randn((8, 256), generator=torch.Generator().manual_seed(2)).cuda()
    check_select(c, bt, q, ctx, seq, top, n_first, n_last)


def test_select_pages_equal_scores_go_by_the_lower_page():
    c, bt = filled(4, 2, 64, [1600], 23)
    k, _ = c.pool.layer_views(0)
    k.fill_(1.0)
    c.index.update(D.dev(bt), D.dev(np.zeros(1, np.int32)), D.dev(np.array([1600], np.int32)), 1600)
    q = torch.randn((3, 256), generator=torch.Generator().manual_seed(3)).cuda()
    q[1] = 0
    pages, _ = check_select(c, bt, q, [1600, 1599, 1200], [0, 0, 0], 9, 1, 2)
    assert pages[0, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 98, 99]


def test_select_pages_queries_of_every_kind():
    c, bt = filled(8, 2, 64, [900], 24)
    q = torch.randn((6, 512), generator=torch.Generator().manual_seed(4))
    q[0, 3], q[0, 100], q[1, 7], q[1, 9] = float("nan"), float("inf"), float("-inf"), 3e38
    q[2] *= 1e-41
    q[3] *= 1e30
    q[4] = 0
    q[5, :64] = 127.0 / 128
    check_select(c, bt, q.cuda(), [900, 890, 880, 870, 860, 850], [0] * 6, 11, 1, 1)


def test_select_pages_huge_keys_and_missing_pages():
    """scores that leave fp32 stop at its largest value; a table without the page scores the lowest"""
    c, bt = filled(2, 1, 64, [640], 25)
    k, _ = c.pool.layer_views(0)
    k.mul_(2.0 ** 120)
    c.index.update(D.dev(bt), D.dev(np.zeros(1, np.int32)), D.dev(np.array([640], np.int32)), 640)
    q = torch.randn((1, 128), generator=torch.Generator().manual_seed(5)).cuda()
    check_select(c, bt, q, [640], [0], 6, 1, 1)
    c, bt = filled(2, 1, 64, [640], 25)
    bt[0, [3, 9]] = [-1, c.blocks]
    pages, _ = B.op_select_pages(c.model, c.pool, c.index, 0, q, D.dev(bt), D.dev(np.array([640], np.int32)), 38, n_first=0, n_last=0)
    assert pages[0, 0].tolist() == [p for p in range(40) if p not in (3, 9)]


def test_select_pages_long_list_and_other_layer():
    lens = [40000, 35001]
    c, bt = filled(2, 2, 64, lens, 26, layers=2, layer=1)
    q = torch.randn((4, 128), generator=torch.Generator().manual_seed(6)).cuda()
    check_select(c, bt, q, [40000, 35001, 20000, 33], [0, 1, 0, 1], 300, 1, 1, layer=1)


# ---- attention over listed pages -----------------------------------------------------------------------------------

def check_attend(c, bt, q, ctx, seq, pages, counts=None, layer=0):
    say("attend", c.n_q, c.n_kv, c.d, "rows", len(ctx), "top", pages.shape[2])
    out = B.op_sparse_attention(c.model, c.pool, layer, q, D.dev(bt), D.dev(np.array(ctx, np.int32)), pages, counts,
                                row_seq=D.dev(np.array(seq, np.int32)))
    got = out.double().cpu().numpy().reshape(len(ctx), c.n_kv, c.G, c.d)
    keys, values = c.keys(layer), c.values(layer)
    qn = q.double().cpu().numpy().reshape(got.shape)
    lists = pages.cpu().numpy()
    cnt = [pages.shape[2]] * len(ctx) if counts is None else counts.cpu().numpy()
    for r in range(len(ctx)):
        for h in range(c.n_kv):
            ks, vs = [np.zeros((0, c.d))], [np.zeros((0, c.d))]
            for p in lists[r, h, :max(0, min(cnt[r], pages.shape[2]))].tolist():
                if 0 <= p and p * 16 < ctx[r]:
                    n = min(16, ctx[r] - p * 16)
                    ks.append(keys[bt[seq[r], p], :n, h])
                    vs.append(values[bt[seq[r], p], :n, h])
            k, v = np.concatenate(ks), np.concatenate(vs)
            want, slack = D.attend(qn[r, h], k, v)
            top = abs(v).max() if len(v) else 0.0
            err = abs(got[r, h] - want).max()
            assert err <= (2 * slack + 2.0 ** -20) * top, (r, h, err, slack, top)
    return out


@pytest.mark.parametrize("heads", ((1, 1, 64), (4, 2, 64), (8, 2, 128), (8, 1, 128), (16, 1, 64), (32, 2, 128), (4, 4, 128), (2, 1, 128), (16, 1, 128)))
@pytest.mark.parametrize("rows", (1, 40))
def test_sparse_attention_head_layouts(heads, rows):
    lens = [1000, 17, 333, 95, 2]
    c, bt = filled(*heads, lens, 31, spread=False)
    seq = [r % 5 for r in range(rows)]
    ctx = [max(0, lens[s] - r // 5) for r, s in enumerate(seq)]
    q = torch.randn((rows, heads[0] * heads[2]), generator=torch.Generator().manual_seed(7)).cuda()
    pages, counts = check_select(c, bt, q, ctx, seq, 33, 1, 1)
    check_attend(c, bt, q, ctx, seq, pages, counts)
    check_attend(c, bt, q, ctx, seq, pages)


@pytest.mark.parametrize("top", (1, 2, 3, 15, 16, 17, 63, 64, 65, 130, 250))
def test_sparse_attention_list_lengths(top):
    c, bt = filled(4, 1, 128, [4000], 32, spread=False)
    q = torch.randn((2, 512), generator=torch.Generator().manual_seed(8)).cuda()
    pages, counts = check_select(c, bt, q, [4000, 3991], [0, 0], top, 0, 1)
    check_attend(c, bt, q, [4000, 3991], [0, 0], pages, counts)


def test_sparse_attention_lists_of_the_callers_own():
    """any order, entries that are no page of the row, counts beyond the list and below zero, rows that see nothing"""
    lens = [200, 37, 16]
    c, bt = filled(8, 2, 64, lens, 33, spread=False)
    ctx, seq = [200, 199, 37, 16, 0, 0, 5, -3], [0, 0, 1, 2, 0, 1, 0, 0]
    lists = np.full((8, 2, 9), -1, np.int32)
    lists[0, 0] = [12, 0, 5, 3, 7, 11, 1, 2, 9]
    lists[0, 1] = [-1, 12, -7, 13, 100000, 2147483647, -2147483648, 4, -1]
    lists[1, 0, :3] = [12, 11, 12 + 1]
    lists[2] = [2, 1, 0, 3, 4, -1, -1, -1, -1]
    lists[3, :, 0] = [0, 1]
    lists[4] = lists[5] = np.arange(9)
    lists[6, :, 4] = 0
    lists[7] = 0
    q = torch.randn((8, 512), generator=torch.Generator().manual_seed(9)).cuda()
    out = check_attend(c, bt, q, ctx, seq, D.dev(lists))
    assert (out.view(8, 8, 64)[3, 4:] == 0).all() and (out[4:6] == 0).all() and (out[7] == 0).all()
    for counts in ([9, 3, 1, 1, 9, 0, 5, 9], [0, 100, -5, 2, 1, 1, 4, 0]):
        check_attend(c, bt, q, ctx, seq, D.dev(lists), D.dev(np.array(counts, np.int32)))


def test_sparse_attention_sharp_and_flat_scores():
    c, bt = filled(4, 2, 128, [3000], 34)
    q = torch.randn((3, 512), generator=torch.Generator().manual_seed(10))
    q[0] *= 30.0
    q[1] *= 1e-6
    pages, counts = check_select(c, bt, q.cuda(), [3000, 2999, 2990], [0, 0, 0], 100, 1, 1)
    check_attend(c, bt, q.cuda(), [3000, 2999, 2990], [0, 0, 0], pages, counts)


def test_sparse_attention_of_all_pages_is_paged_attention():
    lens = [700, 33, 1, 256]
    c, bt = filled(32, 8, 128, lens, 35, spread=False)
    q = torch.randn((4, 4096), generator=torch.Generator().manual_seed(11)).cuda()
    ctx = D.dev(np.array(lens, np.int32))
    pages, counts = B.op_select_pages(c.model, c.pool, c.index, 0, q, D.dev(bt), ctx, 44)
    got = B.op_sparse_attention(c.model, c.pool, 0, q, D.dev(bt), ctx, pages, counts)
    want = B.op_paged_attention(c.model, c.pool, 0, q, D.dev(bt), ctx)
    assert (got - want).abs().max().item() <= 1e-4 * want.abs().max().item()  # that one takes two bf16 terms of q and P


def test_offsets_beyond_32_bits():
    """pages whose tiles and records lie more than 2^32 elements into the pool"""
    d, n_kv = 128, 8
    blocks = (1 << 32) // (n_kv * 2 * 16 * d) + 200
    bt = np.array([list(range(blocks - 60, blocks))], np.int32)
    c, bt = filled(32, n_kv, d, [900], 36, pages=(bt, blocks), spread=False)
    small, bt2 = filled(32, n_kv, d, [900], 36, pages=(np.arange(60, dtype=np.int32)[None], 60), spread=False)
    q = torch.randn((2, 4096), generator=torch.Generator().manual_seed(12)).cuda()
    ctx, seq = D.dev(np.array([900, 850], np.int32)), D.dev(np.zeros(2, np.int32))
    new = torch.randn((10, 1, 8, 128), generator=torch.Generator().manual_seed(13)).cuda()
    for e, t in ((c, bt), (small, bt2)):
        cos, sin = B.rope_table(torch.arange(900, 910, dtype=torch.int32, device="cuda"), 128, 10000.0)
        e.pool.append_rope(0, new[:, 0], new[:, 0], cos, sin, D.dev(t), D.dev(np.array([0, 10], np.int32)), D.dev(np.array([900], np.int32)), index=e.index)
    say("offsets: pool of", c.pool.memory.numel(), "bytes")
    ctx = D.dev(np.array([910, 850], np.int32))
    a = B.op_select_pages(c.model, c.pool, c.index, 0, q, D.dev(bt), ctx, 20, row_seq=seq)
    b = B.op_select_pages(small.model, small.pool, small.index, 0, q, D.dev(bt2), ctx, 20, row_seq=seq)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(B.op_sparse_attention(c.model, c.pool, 0, q, D.dev(bt), ctx, *a, row_seq=seq),
                       B.op_sparse_attention(small.model, small.pool, 0, q, D.dev(bt2), ctx, *b, row_seq=seq))


# ---- verification --------------------------------------------------------------------------------------------------

def check_verify(logits, tokens, uniforms, noise, draft_logits=None, lens=None, temperature=None, strict=True):
    batch, rows, vocab = logits.shape
    say("verify", tuple(logits.shape), "draft", draft_logits is not None, "lens", lens is not None)
    f = lambda t: None if t is None else t.cuda()  # noqa: E731
    out, took, prob = B.verify_drafts(f(logits) if not logits.is_cuda else logits, f(tokens), f(uniforms), f(noise), f(draft_logits),
                                      f(lens), f(temperature))
    out, took, prob = out.cpu().numpy(), took.cpu().numpy(), prob.cpu().numpy()
    lg, dl = logits.cpu().numpy(), None if draft_logits is None else draft_logits.cpu().numpy()
    decided = 0
    for i in range(batch):
        n = rows - 1 if lens is None else min(max(int(lens[i]), 0), rows - 1)
        want, a, pr, near = D.verify(lg[i], tokens[i].numpy(), uniforms[i].numpy(), noise[i].numpy(), None if dl is None else dl[i], n,
                                     1.0 if temperature is None else float(temperature[i]))
        assert (abs(prob[i] - pr) <= 2.0 ** -16 * pr + 1e-37).all(), (i, prob[i], pr)
        if not near:
            decided += 1
            assert took[i] == a and out[i].tolist() == want, (i, out[i], want, took[i], a)
    assert decided >= (batch + 1) // 2 or not strict
    return out, took, prob


def drafts(batch, n, vocab, seed, scale=2.0, noise_scale=0.7):
    g = torch.Generator().manual_seed(seed)
    logits = torch.randn((batch, n + 1, vocab), generator=g) * scale
    draft = logits[:, :n] + noise_scale * torch.randn((batch, n, vocab), generator=g)
    tokens = torch.multinomial(torch.softmax(draft, -1).reshape(batch * n, vocab), 1, generator=g).view(batch, n).int() if n else torch.zeros((batch, 0), dtype=torch.int32)
    return logits, draft, tokens, torch.rand((batch, n), generator=g), torch.empty((batch, vocab)).exponential_(generator=g)


@pytest.mark.parametrize("vocab", (1, 2, 7, 255, 1024, 4095, 4096, 4097, 50257))
@pytest.mark.parametrize("with_draft", (True, False))
def test_verify_vocabularies(vocab, with_draft):
    logits, draft, tokens, u, noise = drafts(9, 3, vocab, vocab)
    check_verify(logits, tokens, u, noise, draft if with_draft else None)


@pytest.mark.parametrize("batch,n", ((1, 0), (5, 0), (1, 1), (3, 1), (2, 16), (1, 127), (70, 2)))
def test_verify_numbers_of_drafts(batch, n):
    logits, draft, tokens, u, noise = drafts(batch, n, 600, 100 + n)
    check_verify(logits, tokens, u * 0.3, noise, draft)
    check_verify(logits, tokens, u, noise, None)


def test_verify_ragged_lengths_and_temperatures():
    logits, draft, tokens, u, noise = drafts(24, 5, 3001, 41)
    lens = torch.tensor([i % 9 - 1 for i in range(24)], dtype=torch.int32)  # -1 and beyond 5 among them
    temp = torch.tensor([0.0, 0.3, 1.0, 2.5, -1.0, 0.7] * 4)
    best = logits[:, :5].argmax(-1).int()
    tokens[::2] = best[::2]
    check_verify(logits, tokens, u, noise, draft, lens, temp)
    check_verify(logits, tokens, u, noise, None, lens, temp)
    check_verify(logits, tokens, u, noise, draft, None, temp)


def test_verify_greedy_ties_go_to_the_lower_token():
    logits = torch.zeros((3, 3, 9000))
    logits[0, :, [5000, 700]] = 3.0
    logits[1, 0, 8999] = 1.0
    tokens = torch.tensor([[700, 5000], [8999, 0], [0, 0]], dtype=torch.int32)
    out, took, _ = check_verify(logits, tokens, torch.full((3, 2), 0.5), torch.ones((3, 9000)), None, None, torch.zeros(3))
    assert out.tolist() == [[700, 700, -1], [8999, 0, 0], [0, 0, 0]] and took.tolist() == [1, 2, 2]


def test_verify_equal_races_go_to_the_lower_token():
    logits = torch.zeros((2, 1, 10000))
    noise = torch.full((2, 10000), 2.0)
    noise[0, [9000, 4100]] = 1.0
    out, _, _ = check_verify(logits, torch.zeros((2, 0), dtype=torch.int32), torch.zeros((2, 0)), noise, strict=False)
    assert out.tolist() == [[4100], [0]]


def test_verify_same_distributions_take_every_draft():
    logits, _, _, u, noise = drafts(6, 4, 2000, 43)
    tokens = torch.multinomial(torch.softmax(logits[:, :4], -1).reshape(24, 2000), 1, generator=torch.Generator().manual_seed(1)).view(6, 4).int()
    _, took, prob = check_verify(logits, tokens, u * 0.999, noise, logits[:, :4].clone())
    assert (took == 4).all() and (prob == 1).all()


def test_verify_logits_of_every_kind():
    logits, draft, tokens, u, noise = drafts(8, 3, 5000, 44)
    inf, nan = float("inf"), float("nan")
    logits[0, :, ::2] = -inf                 # a mask that leaves half the tokens
    tokens[0] = torch.tensor([1, 2, 3])      # token 2 is masked
    logits[1] = -inf                         # nothing left: every p is 0
    logits[2, 0, 17] = inf                   # all of p at one token
    tokens[2, 0] = 17
    logits[3, 1, 100:200] = nan              # NaN counts as masked
    tokens[3] = torch.tensor([5, 150, 6])
    logits[4, 0] = torch.finfo(torch.float32).min
    draft[5, 0, tokens[5, 0].long()] = -inf  # the draft says it cannot be its own token
    draft[6] = -inf
    tokens[7] = torch.tensor([-1, 5000, 2])  # no tokens at all
    for temp in (None, torch.full((8,), 0.5), torch.zeros(8), torch.full((8,), 1e-42)):
        check_verify(logits, tokens, u, noise, draft, None, temp, strict=False)
        out, _, _ = check_verify(logits, tokens, u, noise, None, None, temp, strict=False)
        assert out[1].tolist() == [-1, -1, -1, -1]


def test_verify_what_the_draft_had_is_taken_off():
    """p = (1/2, 1/2), q = (0, 1): rejected draft 1 gives token 0 whatever the noise; drafts that were not sampled likewise"""
    logits = torch.zeros((4, 2, 2))
    draft = torch.tensor([-200.0, 0.0]).expand(4, 1, 2).contiguous()
    noise = torch.tensor([[100.0, 1e-3]] * 4)
    tokens, u = torch.ones((4, 1), dtype=torch.int32), torch.tensor([[0.4], [0.6], [0.9], [0.1]])
    for dl in (draft, None):
        out, took, prob = check_verify(logits, tokens, u, noise, dl, strict=False)
        assert took.tolist() == [1, 0, 0, 1] and out.tolist() == [[1, 1], [0, -1], [0, -1], [1, 1]] and abs(prob - 0.5).max() < 1e-6


def test_verify_row_strides():
    logits, draft, tokens, u, noise = drafts(5, 2, 777, 45)
    wide = torch.full((5, 3, 801), float("nan"))
    wide[:, :, 3:780] = logits
    wd = torch.full((5, 2, 779), float("nan"))
    wd[:, :, 1:778] = draft
    check_verify(wide.cuda()[:, :, 3:780], tokens, u, noise, wd.cuda()[:, :, 1:778])


def test_verify_distribution_is_the_targets():
    """the first token out of verification is distributed as the target's own sample, whatever the draft: chi-square over 8 tokens"""
    batch, n, V = 12000, 2, 8
    g = torch.Generator(device="cuda").manual_seed(5)
    p = torch.tensor([2.0, 1.0, 0.0, 0.5, -1.0, 1.5, 0.2, -3.0], device="cuda")
    qd = torch.tensor([0.0, 2.0, 1.0, -0.5, 1.0, -1.0, 0.3, 0.0], device="cuda")
    logits = p.expand(batch, n + 1, V).contiguous()
    draft = qd.expand(batch, n, V).contiguous()
    tokens = torch.multinomial(torch.softmax(draft, -1).view(-1, V), 1, generator=g).view(batch, n).int()
    u = torch.rand((batch, n), generator=g, device="cuda")
    noise = torch.empty((batch, V), device="cuda").exponential_(generator=g)
    out, took, _ = B.verify_drafts(logits, tokens, u, noise, draft)
    want = torch.softmax(p, -1).double() * batch
    seen = torch.bincount(out[:, 0].long(), minlength=V).double()
    assert ((seen - want) ** 2 / want).sum().item() < 35  # 7 degrees of freedom: one in 10^5
    taken = took >= 1
    second = torch.bincount(out[taken, 1].long(), minlength=V).double()
    want = torch.softmax(p, -1).double() * taken.sum()
    assert ((second - want) ** 2 / want).sum().item() < 35


# ---- 4-bit products ------------------------------------------------------------------------------------------------

def weights(N, K, group, zeros, seed):
    g = torch.Generator().manual_seed(seed)
    w4 = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    scales = (0.5 + torch.rand((N, K // group), generator=g)).to(torch.bfloat16) * torch.where(torch.rand((N, K // group), generator=g) < 0.1, -1, 1)
    z = torch.randint(0, 16, (N, K // group), generator=g, dtype=torch.uint8) if zeros else None
    return w4, scales.to(torch.bfloat16), z


def check_linear4(lin, w, s, x, group, y0=None, accumulate=False):
    M, K = x.shape
    say("linear4", lin.N, K, "group", group, "rows", M, "accumulate", accumulate)
    y = None if y0 is None else y0.cuda()
    got = lin(x.cuda(), y, accumulate).double().cpu().numpy()
    xd = x.double().numpy()
    ok = np.isfinite(xd).all(1)
    xk = np.where(ok[:, None], xd, 0.0)
    want = xk @ w.T + (y0.double().numpy() if accumulate else 0)
    groups = K // group
    blocks = -(-K // 128)
    top = np.abs(np.pad(xk, ((0, 0), (0, blocks * 128 - K)))).reshape(M, blocks, 128).max(2).repeat(128 // group, 1)[:, :groups]
    # the rounding of x: 2^-23 of the largest value of its 128 for each product; sums over the groups in fp32
    digits = (top[:, None, :] * 2.0 ** -23 * abs(w).reshape(1, lin.N, groups, group).sum(3)).sum(2)
    parts = abs(np.einsum("mgk,ngk->mng", xk.reshape(M, groups, group), w.reshape(lin.N, groups, group)))
    sums = (groups + 6) * 2.0 ** -24 * (parts.sum(2) + (abs(y0.double().numpy()) if accumulate else 0))
    # a group's digit sums are joined in fp32 before its zero point's share is off in no digit: nothing to add for it
    err = abs(got - want)[ok]
    assert (err <= (digits + sums)[ok] + 1e-37).all(), (err / (digits + sums)[ok]).max()
    assert np.isnan(got[~ok]).all()
    return got


@pytest.mark.parametrize("group", (32, 64, 128))
@pytest.mark.parametrize("zeros", (False, True))
@pytest.mark.parametrize("N,groups", ((16, 4), (1, 1), (17, 3), (333, 7), (100, 33)))
def test_linear4_shapes(N, groups, group, zeros):
    w4, s, z = weights(N, groups * group, group, zeros, N)
    w, sk = D.weights4(w4, s, z, group)
    lin = B.Linear4(w4.cuda(), s.cuda(), None if z is None else z.cuda())
    for M in (1, 3):
        check_linear4(lin, w, sk, torch.randn((M, groups * group), generator=torch.Generator().manual_seed(M)), group)


@pytest.mark.parametrize("M", (1, 2, 4, 5, 6, 8, 15, 16, 17, 31, 32, 33, 48, 49, 64, 65, 100, 130))
@pytest.mark.parametrize("group,zeros", ((128, False), (64, True), (32, False)))
def test_linear4_rows(M, group, zeros):
    w4, s, z = weights(75, 640, group, zeros, M)
    w, sk = D.weights4(w4, s, z, group)
    lin = B.Linear4(w4.cuda(), s.cuda(), None if z is None else z.cuda())
    x = torch.randn((M, 640), generator=torch.Generator().manual_seed(M))
    x[:, 17] *= 100.0
    check_linear4(lin, w, sk, x, group)
    check_linear4(lin, w, sk, x, group, torch.randn((M, 75), generator=torch.Generator().manual_seed(1)), True)


@pytest.mark.parametrize("N,K,group,M", ((4096, 4096, 128, 1), (2000, 5120, 64, 5), (4100, 2048, 128, 16), (1500, 14336, 128, 33), (9000, 1024, 32, 64), (700, 8192, 32, 7)))
@pytest.mark.parametrize("zeros", (False, True))
def test_linear4_larger(N, K, group, M, zeros):
    w4, s, z = weights(N, K, group, zeros, 3)
    lin = B.Linear4(w4.cuda(), s.cuda(), None if z is None else z.cuda())
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(2))
    got = lin(x.cuda())
    pick = np.r_[0:40, N // 2:N // 2 + 40, N - 40:N]
    w, sk = D.weights4(w4[pick], s[pick], None if z is None else z[pick], group)
    sub = got.cpu()[:, pick]

    class Rows:  # the same check on some of the columns
        def __init__(self):
            self.N = len(pick)

        def __call__(self, x, y, accumulate):
            return sub
    check_linear4(Rows(), w, sk, x, group)


@pytest.mark.parametrize("M", (1, 4, 7, 16, 17))
@pytest.mark.parametrize("group,zeros", ((128, False), (64, True), (32, True)))
def test_linear4_long_rows(M, group, zeros):
    K = 70016 - 70016 % group + group  # more than 16 slices hold at once
    w4, s, z = weights(24, K, group, zeros, 8)
    w, sk = D.weights4(w4, s, z, group)
    lin = B.Linear4(w4.cuda(), s.cuda(), None if z is None else z.cuda())
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(M))
    check_linear4(lin, w, sk, x, group)
    check_linear4(lin, w, sk, x, group, torch.randn((M, 24), generator=torch.Generator().manual_seed(1)), True)


def some_columns(lin, pick):
    """lin as far as check_linear4 goes, of the columns `pick`"""
    class Some:
        N = len(pick)

        def __call__(self, x, y, accumulate):
            whole = None
            if y is not None:
                whole = torch.zeros((x.shape[0], lin.N), device="cuda")
                whole[:, pick] = y
            return lin(x, whole, accumulate)[:, pick]
    return Some()


# rows and sizes that the tiled kernel takes: every height of its tiles, one pass and more
@pytest.mark.parametrize("N,K,group,M", ((8001, 8448, 128, 17), (8001, 8448, 128, 32), (5333, 8448, 128, 48), (4001, 8448, 128, 64), (2700, 8448, 128, 100),
                                         (1900, 8448, 128, 130), (5003, 8480, 32, 17), (3400, 8480, 32, 33), (2507, 8480, 32, 64), (5003, 8512, 64, 20),
                                         (3401, 8512, 64, 40), (2507, 8512, 64, 64), (1700, 8512, 64, 100)))
@pytest.mark.parametrize("zeros", (False, True))
def test_linear4_many_rows(N, K, group, M, zeros):
    w4, s, z = weights(N, K, group, zeros, 12)
    lin = B.Linear4(w4.cuda(), s.cuda(), None if z is None else z.cuda())
    pick = np.r_[0:20, 240:272, N // 2:N // 2 + 20, N - 40:N]
    w, sk = D.weights4(w4[pick], s[pick], None if z is None else z[pick], group)
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(M))
    x[:, 17] *= 100.0
    check_linear4(some_columns(lin, pick), w, sk, x, group)
    check_linear4(some_columns(lin, pick), w, sk, x, group, torch.randn((M, len(pick)), generator=torch.Generator().manual_seed(1)), True)
    flat = torch.zeros(M * K + 1, device="cuda")
    flat[1:] = x.view(-1).cuda()
    assert torch.equal(lin(flat[1:].view(M, K)), lin(x.cuda()))


def test_linear4_many_rows_of_every_kind():
    w4, s, z = weights(2507, 8512, 64, True, 9)
    pick = np.r_[0:64]
    w, sk = D.weights4(w4[pick], s[pick], z[pick], 64)
    lin = B.Linear4(w4.cuda(), s.cuda(), z.cuda())
    some = some_columns(lin, pick)
    x = torch.randn((64, 8512), generator=torch.Generator().manual_seed(4))
    x[0] = 0
    x[0, 100] = 1e-30
    x[1, 64:128] = 0
    x[1, 300] = 1e20
    check_linear4(some, w, sk, x, 64)
    x[0, 5], x[1, 8500] = float("nan"), float("-inf")
    check_linear4(some, w, sk, x, 64)
    x = torch.full((64, 8512), 1e-41)
    assert lin(x.cuda()).abs().max().item() < 1e-36


@pytest.mark.parametrize("M", (3, 7, 12, 20))
def test_linear4_rows_that_are_not_aligned(M):
    w4, s, z = weights(40, 384, 128, False, 5)
    lin = B.Linear4(w4.cuda(), s.cuda())
    flat = torch.randn(M * 384 + 3, generator=torch.Generator().manual_seed(6)).cuda()
    for shift in (1, 2, 3):
        assert torch.equal(lin(flat[shift:shift + M * 384].view(M, 384)), lin(flat[shift:shift + M * 384].view(M, 384).clone()))


@pytest.mark.parametrize("M", (2, 6, 40))
def test_linear4_rows_of_every_kind(M):
    w4, s, z = weights(64, 512, 64, True, 9)
    w, sk = D.weights4(w4, s, z, 64)
    lin = B.Linear4(w4.cuda(), s.cuda(), z.cuda())
    x = torch.randn((M, 512), generator=torch.Generator().manual_seed(4))
    x[0] = 0
    x[0, 100] = 1e-30
    x[1, 64:128] = 0
    x[1, 300] = 1e20
    check_linear4(lin, w, sk, x, 64)
    x[0, 5], x[1, 500] = float("nan"), float("-inf")
    check_linear4(lin, w, sk, x, 64)
    x = torch.full((M, 512), 1e-41)
    assert lin(x.cuda()).abs().max().item() < 1e-36


def test_linear4_is_the_same_for_a_row_whatever_the_batch_up_to_summation_order():
    w4, s, _ = weights(500, 2048, 128, False, 10)
    lin = B.Linear4(w4.cuda(), s.cuda())
    x = torch.randn((64, 2048), generator=torch.Generator().manual_seed(5)).cuda()
    whole = lin(x)
    for M in (1, 5, 9, 33):
        assert (lin(x[:M].contiguous()) - whole[:M]).abs().max().item() <= 40 * 2.0 ** -24 * 2048 ** 0.5 * 10
    assert torch.equal(lin(x), whole)  # and from run to run exactly


# ---- refusals, streams, graphs -------------------------------------------------------------------------------------

def test_refusals():
    c, bt = filled(4, 2, 64, [100], 51, max_batch=4)
    q, btd, ctx = torch.zeros((1, 256), device="cuda"), D.dev(bt), D.dev(np.array([100], np.int32))
    sel = lambda **k: B.op_select_pages(c.model, c.pool, c.index, k.get("layer", 0), k.get("q", q), k.get("bt", btd), k.get("ctx", ctx), k.get("top", 4),  # noqa: E731
                                        n_first=k.get("n_first", 1), n_last=k.get("n_last", 1), row_seq=k.get("row_seq"))
    for bad, code in ((dict(layer=1), -1), (dict(top=0), -1), (dict(n_first=4), -1), (dict(n_first=-1), -1)):
        with pytest.raises(B.ChironError) as e:
            sel(**bad)
        assert e.value.code == code, bad
    five = D.dev(np.zeros(5, np.int32))
    with pytest.raises(B.ChironError) as e:
        sel(q=torch.zeros((5, 256), device="cuda"), ctx=five, row_seq=five)
    assert e.value.code == -3
    with pytest.raises(ValueError):
        sel(q=torch.zeros((1, 128), device="cuda"))
    with pytest.raises(ValueError):
        sel(bt=btd[:, :-1].contiguous())
    with pytest.raises(TypeError):
        sel(q=q.double())
    with pytest.raises(TypeError):
        sel(top=1.5)
    with pytest.raises(ValueError):
        B.op_sparse_attention(c.model, c.pool, 0, q, btd, ctx, torch.zeros((1, 3, 4), dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        B.op_sparse_attention(c.model, c.pool, 0, q, btd, ctx, torch.zeros((1, 2, 4), dtype=torch.int64, device="cuda"))
    other = D.Cache(4, 2, 128, 5)
    with pytest.raises(B.ChironError) as e:
        B.op_select_pages(c.model, c.pool, other.index, 0, q, btd, ctx, 4)
    assert e.value.code == -1 and "another pool" in str(e.value)
    with pytest.raises(B.ChironError) as e:
        B.KVIndex(c.pool, memory=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -5
    k = torch.zeros((3, 2, 64), device="cuda")
    cs = torch.zeros((3, 32), device="cuda")
    st, sl = D.dev(np.array([0, 3], np.int32)), D.dev(np.array([0], np.int32))
    app = lambda **a: c.pool.append_rope(a.get("layer", 0), a.get("k", k), a.get("v", k), a.get("cos", cs), cs, btd, a.get("st", st), sl,  # noqa: E731
                                         q=a.get("q"), index=a.get("index"), q_out=a.get("q_out"))
    for bad, err in ((dict(layer=3), B.ChironError), (dict(k=k.half()), TypeError), (dict(v=k.bfloat16()), TypeError), (dict(v=k[:2]), ValueError),
                     (dict(cos=cs[:2]), ValueError), (dict(st=sl), ValueError), (dict(k=k.transpose(1, 2)), ValueError), (dict(layer=0.5), TypeError),
                     (dict(k=torch.zeros((3, 64, 2), device="cuda").transpose(1, 2)), TypeError), (dict(index=other.index), B.ChironError),
                     (dict(q=k, q_out=torch.zeros((3, 1, 64), device="cuda")), ValueError), (dict(k=k.cpu()), TypeError)):
        with pytest.raises(err):
            app(**bad)
    lg, tk, u, nz = torch.zeros((2, 3, 50), device="cuda"), torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros((2, 2), device="cuda"), torch.ones((2, 50), device="cuda")
    for bad, err in ((dict(t=tk[:, :1].contiguous()), ValueError), (dict(n=nz[:, :49].contiguous()), ValueError), (dict(t=tk.long()), TypeError), (dict(l=lg.half()), TypeError),
                     (dict(d=lg), ValueError), (dict(l=lg.transpose(0, 1).contiguous().transpose(0, 1)), TypeError)):
        with pytest.raises(err):
            B.verify_drafts(bad.get("l", lg), bad.get("t", tk), u, bad.get("n", nz), bad.get("d"))
    with pytest.raises(B.ChironError) as e:
        B.verify_drafts(torch.zeros((1, 129, 4), device="cuda"), torch.zeros((1, 128), dtype=torch.int32, device="cuda"), torch.zeros((1, 128), device="cuda"), torch.ones((1, 4), device="cuda"))
    assert e.value.code == -2
    w4, s, z = weights(8, 128, 64, True, 1)
    for args, err in (((w4[:, :60], s, z), B.ChironError), ((w4, s[:4], z), ValueError), ((w4, s, z[:, :1]), ValueError), ((w4, s.float(), z), TypeError), ((w4.cpu(), s, z), TypeError)):
        with pytest.raises(err):
            B.Linear4(*[t.cuda().contiguous() if i or err is not TypeError or t is not w4 else t for i, t in enumerate(args)])
    with pytest.raises(B.ChironError) as e:
        B.Linear4(w4.cuda(), s[:, :1].repeat(1, 8).contiguous().cuda())  # groups of 16
    assert e.value.code == -2
    lin = B.Linear4(w4.cuda(), s.cuda(), z.cuda())
    x = torch.zeros((2, 128), device="cuda")
    for a, err in (((x[:, :64].contiguous(),), ValueError), ((x.double(),), TypeError), ((x, None, True), ValueError), ((x, torch.zeros((1, 8), device="cuda")), ValueError),
                   ((x, x.view(-1)[:16].view(2, 8)), B.ChironError)):
        with pytest.raises(err):
            lin(*a)
    assert lin(x[:0]).shape == (0, 8)


def test_on_another_stream_and_in_a_graph():
    """the operators run on the current stream; captured, a replay reads what the inputs hold then"""
    c, bt = filled(8, 2, 64, [500, 300], 61, spread=False)
    btd, ctx = D.dev(bt), D.dev(np.array([500, 300], np.int32))
    g = torch.Generator().manual_seed(3)
    qs = [torch.randn((2, 512), generator=g).cuda() for _ in range(3)]
    w4, s, _ = weights(512, 512, 128, False, 2)
    lin = B.Linear4(w4.cuda(), s.cuda())
    logits, draft, tokens, u, noise = (t.cuda() for t in drafts(2, 2, 1000, 7))
    q = qs[0].clone()

    def work():
        y = lin(q)
        pages, counts = B.op_select_pages(c.model, c.pool, c.index, 0, y, btd, ctx, 9)
        o = B.op_sparse_attention(c.model, c.pool, 0, y, btd, ctx, pages, counts)
        return (y, pages, counts, o) + B.verify_drafts(logits, tokens, u, noise, draft)

    want = []
    for x in qs:
        q.copy_(x)
        want.append([t.clone() for t in work()])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for x, w in zip(qs, want):
            q.copy_(x)
            got = work()
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, w))
    torch.cuda.current_stream().wait_stream(side)
    say("graph capture")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for x, w in zip(qs + qs, want + want):
        q.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, w))
        work()
        torch.cuda.synchronize()
