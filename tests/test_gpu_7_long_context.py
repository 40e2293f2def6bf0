"""The long-context operators on the GPU against their definitions in 64 bits: page lists, the cache in 8 bits, attention of new rows within
windows.  Needs a real MI355X: run with -m gpu.

Tolerances.  Whole numbers are equal.  What the 8-bit cache holds follows exactly from keys that are rotated in fp32 with every operation
rounded, which numpy does alike: it is equal too.  Attention: logits that are off by at most s move an average of values by at most 2 s max|v|,
with s from the products' own magnitudes; the exponentials 2^-20 and the fp32 sums of n weights over four lanes and a tree, of weights
and of weighted values, (n / 4 + 40) 2^-24 each.  With bf16 queries a weight is rounded to bf16, 2^-8 of itself and so at most 2^-8 of the
weighted average of |v|, and the result by 2^-8 of itself."""
import ctypes as C

import numpy as np
import pytest
import torch

import long_context as L
from paper_2501_08090_amd import binding as B

pytestmark = pytest.mark.gpu
PAGE = 16


def say(*a):
    print(*a, flush=True)


def ints(a):
    return L.dev(np.asarray(a, np.int32))


# ---- page lists --------------------------------------------------------------------------------------------------------

def table_case(batch, width, seed, drafts=3, prompts=0.1, free=1.0):
    rng = np.random.default_rng(seed)
    top = width * PAGE
    keep = rng.integers(0, max(1, top - drafts - 1), batch) * (rng.random(batch) < 0.85)
    new = np.where(rng.random(batch) < prompts, rng.integers(0, top // 2 + 1, batch), rng.integers(0, drafts + 1, batch))
    has = -(-np.minimum(top, keep + drafts) // PAGE)
    ids = rng.permutation(int(has.sum()) + 8 * batch + 7)
    bt, o = np.full((batch, width), -1, np.int32), 0
    for i, h in enumerate(has):
        bt[i, :h] = ids[o:o + h]
        o += h
    spare = ids[o:o + int(free * 8 * batch) + 1].astype(np.int32)
    pages = np.full(len(ids), -7, np.int32)
    pages[:len(spare)] = spare
    return bt, pages, len(spare), keep.astype(np.int32), new.astype(np.int32)


def check_list(lst, pages):
    n = int(lst.count[0])
    assert n == len(pages) and lst.pages[:n].tolist() == list(pages)


def check_grant(m, bt_gpu, bt, lst, pages, old, new, rows):
    left, starts, seq, pos, slots, granted = L.grant(bt, pages, old, new, rows)
    check_list(lst, left)
    assert np.array_equal(bt_gpu.cpu().numpy(), bt)
    for got, want in zip(m, (starts, seq, pos, slots, granted)):
        assert np.array_equal(got.cpu().numpy(), want)
    return left


@pytest.mark.parametrize("batch,width,free,rows_share", (
    (1, 1, 1.0, 1.0), (1, 40, 1.0, 1.0), (7, 5, 1.0, 1.0), (64, 33, 0.02, 1.0), (65, 17, 1.0, 0.4), (200, 9, 0.05, 0.7), (1024, 3, 0.3, 1.0),
    (1025, 3, 1.0, 0.9), (1501, 130, 0.2, 1.0), (2500, 4, 0.01, 0.5), (3, 2000, 1.0, 1.0), (130, 600, 0.5, 1.0),
    (64, 512, 0.3, 1.0), (63, 521, 0.3, 0.8), (1024, 33, 0.3, 1.0), (5000, 2, 0.5, 0.9), (1000, 32, 1.0, 1.0)))
def test_pages(batch, width, free, rows_share):
    bt, pages, n, keep, new = table_case(batch, width, batch * 7 + width, free=free)
    rows = int(rows_share * new.sum()) + 3
    say("pages", batch, width, "rows", rows, "free", n)
    lst = B.PageList(L.dev(pages), ints([n]))
    gpu = L.dev(bt)
    want = [int(x) for x in pages[:n]]
    lst.release(gpu, L.dev(keep))
    torch.cuda.synchronize()
    want = L.release(bt, want, keep)
    check_list(lst, want)
    assert np.array_equal(gpu.cpu().numpy(), bt)
    m = lst.grant(gpu, L.dev(keep), L.dev(new), rows)
    torch.cuda.synchronize()
    want = check_grant(m, gpu, bt, lst, want, keep, new, rows)
    # again on its own result: the same rows; those that had to wait for pages may find some now
    m = lst.grant(gpu, L.dev(keep), L.dev(new), rows)
    want = check_grant(m, gpu, bt, lst, want, keep, new, rows)
    # what a window has passed
    rng = np.random.default_rng(batch)
    first, end = rng.integers(-5, 40, batch).astype(np.int32), rng.integers(-20, width * PAGE + 50, batch).astype(np.int32)
    lst.release(gpu, L.dev(first), L.dev(end))
    want = L.release(bt, want, first, end)
    check_list(lst, want)
    assert np.array_equal(gpu.cpu().numpy(), bt)


@pytest.mark.parametrize("batch", (5, 1100))
def test_pages_edges(batch):
    """lengths out of range, a list that is empty or full, counts out of range, no rows, requests without new tokens"""
    width = 4
    bt = np.full((batch, width), -1, np.int32)
    old = np.zeros(batch, np.int32)
    new = np.ones(batch, np.int32)
    old[:4], new[:4] = (-1, 5, 2 ** 31 - 1, 63), (3, -2, 2 ** 31 - 1, 1)
    pages = np.arange(3 * batch, dtype=np.int32)
    for count, rows in ((0, 100), (3 * batch, 0), (3 * batch, 5000), (10 ** 6, 5000), (-9, 5000)):
        lst, gpu, want = B.PageList(L.dev(pages), ints([count])), L.dev(bt), bt.copy()
        there = list(range(min(max(count, 0), 3 * batch)))
        m = lst.grant(gpu, L.dev(old), L.dev(new), rows)
        torch.cuda.synchronize()
        check_grant(m, gpu, want, lst, there, old, new, rows)
    # a list with room for two: the other pages stay
    lst, gpu = B.PageList(ints([0] * 6), ints([4])), L.dev(np.arange(batch * width, dtype=np.int32).reshape(batch, width) + 50)
    lst.release(gpu, ints([0] * batch))
    torch.cuda.synchronize()
    assert lst.pages.tolist() == [0, 0, 0, 0, 50, 51] and int(lst.count[0]) == 6
    assert gpu.flatten().tolist() == [-1, -1] + list(range(52, 50 + batch * width))
    # nobody
    m = lst.grant(gpu[:0], ints([]), ints([]), 3)
    lst.release(gpu[:0], ints([]))
    assert m.row_starts.tolist() == [0] and m.row_seq.tolist() == [-1] * 3 and m.slots.tolist() == [-1] * 3 and m.pos.tolist() == [0] * 3
    assert int(lst.count[0]) == 6


# ---- the cache in 8 bits -------------------------------------------------------------------------------------------------

def turned32(x, cos, sin):
    """the rotation with every operation rounded to fp32"""
    a, b = np.split(x.astype(np.float32), 2, -1)
    c, s = cos[:, None], sin[:, None]
    return np.concatenate((a * c - b * s, b * c + a * s), -1)


def check_append8(n_q, n_kv, d, old, new, dtype, fmt, seed, layer=0, layers=1, shift=0, scale=None, special=False, spare_rows=0):
    rng = np.random.default_rng(seed)
    total = [a + b for a, b in zip(old, new)]
    bt, blocks = L.tables(total, seed)
    bt = L.widen(bt, bt.shape[1] + 1)
    c = L.Cache(n_kv, d, blocks, fmt, layers)
    c.fill(bt, old, rng, layer)
    before = [t.clone().view(torch.uint8) for t in c.pool.layer_views(layer)]
    elsewhere = c.pool.memory.clone()
    kb, vb = c.values(layer)
    eb = before[2].view(torch.int8).cpu().numpy().astype(int)
    rows = sum(new) + spare_rows
    fused = rng.standard_normal((rows, (n_q + 2 * n_kv) * d + shift + 8))
    fused *= scale if scale is not None else 2.0 ** rng.integers(-3, 4, (rows, 1))
    if special:
        fused[rng.integers(0, rows, 3), rng.integers(n_q * d, fused.shape[1], 3)] = (np.nan, np.inf, -1e39)
    fused = torch.from_numpy(fused).to(dtype).cuda()
    q = fused[:, shift:shift + n_q * d].unflatten(1, (n_q, d))
    k = fused[:, shift + n_q * d:shift + (n_q + n_kv) * d].unflatten(1, (n_kv, d))
    v = fused[:, shift + (n_q + n_kv) * d:shift + (n_q + 2 * n_kv) * d].unflatten(1, (n_kv, d))
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    pos = np.concatenate([np.arange(a, a + b) for a, b in zip(old, new)] + [np.zeros(spare_rows)]).astype(np.int32)
    cos, sin = B.rope_table(L.dev(pos), d, 10000.0)
    say("append8", fmt, n_q, n_kv, d, dtype, "old", old, "new", new, "shift", shift)
    got_q = c.pool.append_rope(layer, k, v, cos, sin, L.dev(bt), L.dev(starts), ints(old), q=q)
    torch.cuda.synchronize()
    cos, sin = cos.cpu().numpy(), sin.cpu().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        wq, wk = turned32(q.float().cpu().numpy(), cos, sin), turned32(k.float().cpu().numpy(), cos, sin)
    wv = v.float().cpu().numpy()
    assert np.array_equal(got_q.cpu().numpy(), wq, equal_nan=True)
    ka, va = c.values(layer)
    ea = c.pool.layer_views(layer)[2].cpu().numpy().astype(int)
    touched = np.zeros((blocks, PAGE), bool)
    written = np.zeros(blocks, bool)
    for i, (o, n) in enumerate(zip(old, new)):
        for pg in range(o // PAGE, -(-(o + n) // PAGE) if n else 0):
            a, b, block = max(o - pg * PAGE, 0), min(o + n - pg * PAGE, PAGE), bt[i, pg]
            src = slice(starts[i] + pg * PAGE + a - o, starts[i] + pg * PAGE + b - o)
            touched[block, :b] = True
            written[block] = True
            for h in range(n_kv):
                for after, had, x, j in ((ka, kb, wk, 0), (va, vb, wv, 1)):
                    want, e = L.store(had[block, :a, h], eb[block, h, j], x[src, h], fmt)
                    assert ea[block, h, j] == e, (i, pg, h, j)
                    assert np.array_equal(after[block, :b, h], want), (i, pg, h, j)
    # nothing else moved: other slots' codes, other pages' exponents, other layers
    for t, was in zip(c.pool.layer_views(layer)[:2], before):
        same = (t.view(torch.uint8) == was).reshape(blocks, PAGE, -1).all(2).cpu().numpy()
        assert (same | touched).all()
    assert np.array_equal(ea[~written], eb[~written])
    size = c.pool.memory.numel() // layers
    for l in range(layers):
        if l != layer:
            assert torch.equal(c.pool.memory[l * size:(l + 1) * size], elsewhere[l * size:(l + 1) * size])
    # and the read-back gives the same
    look = [(i, p) for i, n in enumerate(total) for p in range(n)] + [(0, -1), (0, bt.shape[1] * PAGE), (0, bt.shape[1] * PAGE - 1)]
    gk, gv = c.pool.gather(layer, L.dev(bt), ints([i for i, _ in look]), ints([p for _, p in look]))
    for j, (i, p) in enumerate(look):
        block = bt[i, p // PAGE] if 0 <= p < bt.shape[1] * PAGE else -1
        for got, have in ((gk, ka), (gv, va)):
            want = have[block, p % PAGE] if block >= 0 else np.zeros((n_kv, d))
            if j < 40 or j >= len(look) - 40:
                assert np.array_equal(got[j].double().cpu().numpy(), want)


@pytest.mark.parametrize("fmt", ("int8", "e4m3"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("n_q,n_kv,d,old,new", (
    (4, 1, 64, [0], [1]), (4, 1, 128, [15], [1]), (2, 2, 64, [16], [1]), (8, 2, 128, [3], [13]), (8, 2, 64, [3], [14]),
    (4, 4, 128, [0, 7, 16, 31, 100], [1, 1, 1, 1, 1]), (6, 3, 64, [0, 7, 16, 31, 5, 40], [16, 40, 0, 1, 3, 77]),
    (16, 8, 128, [0, 250, 33], [65, 129, 1])))
def test_append8(fmt, dtype, n_q, n_kv, d, old, new):
    check_append8(n_q, n_kv, d, old, new, dtype, fmt, seed=len(old) * 10 + d)


@pytest.mark.parametrize("fmt", ("int8", "e4m3"))
@pytest.mark.parametrize("kw", (dict(layer=1, layers=3), dict(shift=3), dict(shift=1, special=True), dict(scale=1e-37), dict(scale=1e36, special=True),
                                dict(scale=0.0), dict(spare_rows=5)))
def test_append8_rows_and_values(fmt, kw):
    check_append8(4, 2, 64, [5, 0, 18], [9, 20, 2], torch.float32, fmt, seed=77, **kw)
    check_append8(4, 1, 128, [5, 30], [4, 3], torch.bfloat16, fmt, seed=78, **kw)


@pytest.mark.parametrize("fmt", ("int8", "e4m3"))
def test_append8_token_by_token(fmt):
    """a page that fills one token at a time: the power of two only grows, and every value is within a step of what was appended"""
    rng = np.random.default_rng(5)
    d, n_kv = 64, 2
    c = L.Cache(n_kv, d, 4, fmt)
    bt = ints([[2, 0]])
    x = rng.standard_normal((20, n_kv, d)) * 2.0 ** rng.integers(-6, 7, (20, 1, 1))
    held = [[np.zeros((0, d)), 0] for _ in range(2 * n_kv)]
    one, zero = torch.ones((1, d // 2), device="cuda"), torch.zeros((1, d // 2), device="cuda")
    for t in range(20):
        k, v = (torch.from_numpy(x[t:t + 1] * s).float().cuda() for s in (1.0, -2.5))
        c.pool.append_rope(0, k, v, one, zero, bt, ints([0, 1]), ints([t]))
        if t % PAGE == 0:
            held = [[np.zeros((0, d)), 0] for _ in range(2 * n_kv)]
        vals, e = c.values(), c.pool.layer_views(0)[2].cpu().numpy()
        for j, src in enumerate((k, v)):
            for h in range(n_kv):
                s = held[j * n_kv + h]
                s[0], s[1] = L.store(s[0], s[1], src[:, h].double().cpu().numpy(), fmt)
                block = 2 if t < PAGE else 0
                assert e[block, h, j] == s[1] and np.array_equal(vals[j][block, :t % PAGE + 1, h], s[0])


def test_append8_skips_what_is_no_page():
    """entries out of the pool, positions behind the table, requests without rows"""
    c = L.Cache(1, 64, 3, "int8")
    before = c.pool.memory.clone()
    k = torch.randn((40, 1, 64), device="cuda")
    cos, sin = B.rope_table(ints(range(40)), 64, 10000.0)
    c.pool.append_rope(0, k, k, cos, sin, ints([[-1, 3], [99, -5]]), ints([0, 20, 40]), ints([0, 30]))
    c.pool.append_rope(0, k, k, cos, sin, ints([[0, 1], [2, 1]]), ints([0, 0, 40]), ints([0, 32]))
    torch.cuda.synchronize()
    assert torch.equal(c.pool.memory, before)


# ---- attention of new rows -------------------------------------------------------------------------------------------------

def check_rows(n_q, n_kv, d, old, new, fmt, dtype, window=0, sinks=0, seed=0, layer=0, layers=1, max_new=None, spare_rows=0, drop=(), stride=0, hot=1.0,
               clip=None):
    """drop: (request, page) whose entry becomes -1, clip: columns of the table"""
    rng = np.random.default_rng(seed)
    total = [a + b for a, b in zip(old, new)]
    bt, blocks = L.tables(total, seed)
    bt = L.widen(bt, bt.shape[1] + 1)
    c = L.Cache(n_kv, d, blocks, fmt, layers)
    c.fill(bt, total, rng, layer)
    for i, p in drop:
        bt[i, p] = blocks + 3 if (i + p) % 2 else -1
    if clip is not None:
        bt = np.ascontiguousarray(bt[:, :clip])
    rows = sum(new) + spare_rows
    x = torch.from_numpy(rng.standard_normal((rows, n_q * d + stride)) * 1.5 * hot).to(dtype).cuda()
    q = x[:, :n_q * d].unflatten(1, (n_q, d))
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    say("rows", fmt, dtype, "heads", n_q, n_kv, d, "old", old, "new", new, "window", window, sinks, "max_new", max_new)
    out = torch.full((rows, n_q, d), 7.5, dtype=dtype, device="cuda")
    got = B.op_row_attention(c.pool, layer, q, L.dev(bt), L.dev(starts), ints(old), window=window, n_sinks=sinks, max_new=max_new, out=out)
    torch.cuda.synchronize()
    assert got is out
    got = out.double().cpu().numpy()
    qd, G = q.double().cpu().numpy(), n_q // n_kv
    kd, vd = c.values(layer)
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    worst = 0.0
    for i, (o, n) in enumerate(zip(old, new)):
        t = np.arange(total[i])
        cols = t // PAGE
        entry = np.where(cols < bt.shape[1], bt[i, np.minimum(cols, bt.shape[1] - 1)], -1)
        there = (entry >= 0) & (entry < blocks)
        k, v = (np.where(there[:, None, None], a[np.where(there, entry, 0), t % PAGE], 0.0) for a in (kd, vd))
        for j in range(n):
            r = starts[i] + j
            if max_new is not None and j >= max_new:
                assert (got[r] == 7.5).all()
                continue
            see = L.visible(o + j, total[i], window, sinks) & there
            vmax = abs(v[see]).max() if see.any() else 0.0
            for h in range(n_kv):
                want, slack = L.attend(qd[r, h * G:(h + 1) * G], k[:, h], v[:, h], see)
                tol = vmax * (2 * slack + 2.0 ** -19 + 2 * (see.sum() / 4 + 40) * 2.0 ** -24)
                if dtype == torch.bfloat16:
                    mean, _ = L.attend(qd[r, h * G:(h + 1) * G], k[:, h], abs(v[:, h]), see)
                    tol = tol + 2.0 ** -8 * mean
                tol = tol + step * abs(want)
                err = abs(got[r, h * G:(h + 1) * G] - want)
                assert (err <= tol).all(), (i, j, h, float((err - tol).max()))
                worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
    assert (got[starts[-1]:] == 7.5).all()
    say("   worst error %.3f of what is allowed" % worst)


GEOMETRIES = ((4, 1, 128), (8, 8, 64), (16, 2, 64), (16, 1, 128), (6, 2, 64), (10, 2, 128), (32, 8, 128))


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("n_q,n_kv,d", GEOMETRIES)
def test_single_tokens(fmt, dtype, n_q, n_kv, d):
    old = [0, 1, 15, 16, 17, 31, 130, 700, 1023]
    for window, sinks in ((0, 0), (1, 0), (16, 1), (40, 17), (300, 4), (5000, 3)):
        check_rows(n_q, n_kv, d, old, [1] * len(old), fmt, dtype, window, sinks, seed=window)


@pytest.mark.parametrize("fmt", ("bf16", "e4m3", "int8"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("n_q,n_kv,d", GEOMETRIES)
def test_few_tokens(fmt, dtype, n_q, n_kv, d):
    old, new = [0, 3, 15, 64, 65, 500, 0], [5, 0, 2, 4, 1, 3, 1]
    for window, sinks in ((0, 0), (1, 2), (3, 0), (33, 5), (200, 20)):
        check_rows(n_q, n_kv, d, old, new, fmt, dtype, window, sinks, seed=window + 1)


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("n_q,n_kv,d", GEOMETRIES[:6])
def test_prompts(fmt, dtype, n_q, n_kv, d):
    old, new = [0, 3, 100, 0, 64, 900], [70, 0, 129, 1, 33, 5]
    for window, sinks in ((0, 0), (1, 0), (17, 3), (100, 40)):
        check_rows(n_q, n_kv, d, old, new, fmt, dtype, window, sinks, seed=window + 2)


@pytest.mark.parametrize("fmt", ("bf16", "int8"))
def test_prompt_sizes(fmt):
    for n in (9, 16, 31, 32, 33, 127, 128, 300):
        check_rows(8, 2, 64, [0, 13], [n, 1], fmt, torch.bfloat16, window=0 if n % 2 else 50, sinks=2, seed=n)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("fmt", ("bf16", "e4m3"))
def test_long(fmt, dtype):
    """shares of several hundred pages, passes in many shares, prompts whose pages are dealt out"""
    check_rows(4, 1, 128, [20000], [1], fmt, dtype, seed=1)
    check_rows(4, 1, 128, [20000, 3, 9000], [2, 1, 5], fmt, dtype, window=7777, sinks=31, seed=2)
    check_rows(4, 1, 64, [5000], [40], fmt, dtype, seed=3)
    check_rows(4, 1, 64, [5000, 1], [40, 20], fmt, dtype, window=2500, sinks=3, seed=4)


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
@pytest.mark.parametrize("n_q,n_kv,d,new", ((32, 8, 128, 1), (8, 8, 64, 1), (16, 2, 64, 1), (8, 4, 128, 2), (8, 2, 128, 40)))
def test_weights_add_up(fmt, n_q, n_kv, d, new):
    """Values that are all 1: what is divided is the divisor, whatever the scores.  n weights, none below 0, are added with n roundings at most on
    either side, the three terms of a weight and the term groups with three more, and the quotient has two: (2n + 8) 2^-24."""
    rng = np.random.default_rng(n_q + d + new)
    old = (np.arange(64) % 15 + 1).tolist()
    total = [o + new for o in old]
    bt, blocks = L.tables(total, 5)
    c = L.Cache(n_kv, d, blocks, fmt)
    n = sum(total)
    k = torch.from_numpy(rng.standard_normal((n, n_kv, d))).float().cuda()
    starts = np.concatenate([[0], np.cumsum(total)]).astype(np.int32)
    cos, sin = torch.ones((n, d // 2), device="cuda"), torch.zeros((n, d // 2), device="cuda")
    c.pool.append_rope(0, k, torch.ones_like(k), cos, sin, L.dev(bt), L.dev(starts), ints([0] * 64))
    rows = np.arange(65, dtype=np.int32) * new
    for scale in (0.5, 1.5, 3.0):
        q = torch.from_numpy(rng.standard_normal((64 * new, n_q, d)) * scale).float().cuda()
        say("weights", fmt, n_q, n_kv, d, new, scale)
        got = B.op_row_attention(c.pool, 0, q, L.dev(bt), L.dev(rows), ints(old), max_new=new).double().cpu().numpy()
        seen = np.concatenate([o + 1 + np.arange(new) for o in old])
        err = abs(got - 1.0).max(axis=(1, 2))
        assert (err <= (2 * seen + 8) * 2.0 ** -24).all(), float((err / ((2 * seen + 8) * 2.0 ** -24)).max())


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_tokens_on_both_sides_of_a_prompt(fmt, dtype):
    """every count of passes up to the first tiles, in calls of few and of many requests (which draw that line elsewhere)"""
    for n_q, n_kv, d in ((4, 1, 128), (16, 2, 64)):
        tg = 16 // (n_q // n_kv)
        new = [tg * p + e for p in (1, 2, 4, 8) for e in (0, 1)] + [1, 8 * tg - 1]
        old = [40 * i + 7 for i in range(len(new))]
        check_rows(n_q, n_kv, d, old, new, fmt, dtype, window=90, sinks=18, seed=21)
        check_rows(n_q, n_kv, d, old * 4, new * 4, fmt, dtype, seed=22)
        check_rows(n_q, n_kv, d, old[-1:], new[7:8], fmt, dtype, seed=23)


@pytest.mark.parametrize("fmt", ("bf16", "int8"))
def test_one_request_in_padded_rows(fmt):
    """the rows' count and what is promised about it say more than the request has"""
    for new in (0, 1, 5, 50):
        check_rows(4, 1, 128, [50], [new], fmt, torch.bfloat16, spare_rows=299, seed=new)
        check_rows(4, 1, 128, [700], [new], fmt, torch.float32, window=100, sinks=3, max_new=200, spare_rows=299, seed=new + 1)


@pytest.mark.parametrize("batch", (63, 64, 65, 200))
def test_many_requests(batch):
    rng = np.random.default_rng(batch)
    old, new = rng.integers(0, 60, batch).tolist(), rng.integers(0, 3, batch).tolist()
    check_rows(4, 2, 64, old, new, "int8", torch.float32, seed=batch)
    new[7], new[batch - 1] = 40, 35
    check_rows(4, 2, 64, old, new, "bf16", torch.float32, window=20, sinks=1, seed=batch + 1)


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_pages_that_are_not_there(fmt, dtype):
    """entries that are no page of the pool, in and out of the window; tables that end before the positions do; rows that see nothing"""
    check_rows(4, 2, 64, [100, 40, 0], [1, 2, 3], fmt, dtype, drop=((0, 2), (1, 0), (1, 1), (1, 2), (2, 0)), seed=1)
    check_rows(4, 2, 64, [100, 40, 0], [30, 20, 40], fmt, dtype, drop=((0, 2), (0, 7), (2, 0), (2, 1)), seed=2)
    check_rows(4, 2, 64, [100, 300], [1, 1], fmt, dtype, window=20, sinks=3, drop=tuple((i, p) for i in (0, 1) for p in range(1, 5)), seed=3)
    check_rows(4, 2, 64, [100, 10, 47], [1, 1, 4], fmt, dtype, window=20, clip=3, seed=4)
    check_rows(4, 2, 64, [30, 10, 90], [50, 1, 20], fmt, dtype, window=16, clip=3, seed=5)


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_queries_that_end_where_their_memory_does(fmt, dtype):
    """the last rows of an allocation of its own, of heads that do not fill the columns of a pass: the same as anywhere else"""
    rng = np.random.default_rng(31)
    for n_q, n_kv, d in ((16, 8, 128), (8, 8, 64), (6, 2, 64), (10, 2, 128), (7, 1, 64)):
        for new in (1, 3, 40):
            old = [31 + i for i in range(10)]
            total = [o + new for o in old]
            bt, blocks = L.tables(total, 3)
            c = L.Cache(n_kv, d, blocks, fmt)
            c.fill(bt, total, rng)
            n = 10 * new * n_q * d
            q = torch.from_numpy(rng.standard_normal(n)).to(dtype).cuda()
            memory = torch.zeros((32 << 20) // q.element_size(), dtype=dtype, device="cuda")  # whole pages of the allocator, and nothing behind
            memory[-n:] = q
            starts = ints(np.arange(11) * new)
            say("end", fmt, dtype, n_q, n_kv, d, new)
            want = B.op_row_attention(c.pool, 0, q.view(-1, n_q, d), L.dev(bt), starts, ints(old), window=38, max_new=new)
            got = B.op_row_attention(c.pool, 0, memory[-n:].view(-1, n_q, d), L.dev(bt), starts, ints(old), window=38, max_new=new)
            torch.cuda.synchronize()
            assert torch.equal(got, want)
            del memory


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
def test_row_starts_that_do_not_ascend(fmt):
    """more requests claim rows than there are: nothing is written but rows of out and the workspace"""
    n_q, n_kv, d, batch, rows = 8, 2, 64, 200, 4
    c = L.Cache(n_kv, d, batch, fmt)
    bt = ints(np.arange(batch).reshape(batch, 1))
    k = torch.ones((batch * 16, n_kv, d), device="cuda")
    c.pool.append_rope(0, k, k, torch.ones((batch * 16, d // 2), device="cuda"), torch.zeros((batch * 16, d // 2), device="cuda"), bt,
                       ints(np.arange(batch + 1) * 16), ints([0] * batch))
    for dtype in (torch.float32, torch.bfloat16):
        for starts in ([0, 4] * 100 + [0], [0, 1] * 100 + [0], [0, 4, 0, 2] * 50 + [4], [-1, 3] * 100 + [9], [4] * 201, [3, 2, 1, 0] * 50 + [4]):
            for max_new in (4, 1):
                say("starts", fmt, dtype, starts[:5], max_new)
                q = torch.ones((rows, n_q, d), dtype=dtype, device="cuda")
                out = torch.full((3 * rows, n_q, d), 7.5, dtype=dtype, device="cuda")
                need = B.load().chiron_row_attention_workspace_bytes(n_q, n_kv, d, batch, rows, max_new)
                work = torch.full((need + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
                table, old = ints(starts), ints([12] * batch)
                a = B.AttnRows(q.data_ptr(), out[rows:2 * rows].data_ptr(), n_q * d, B.CHIRON_F32 if dtype == torch.float32 else B.CHIRON_BF16, n_q, bt.data_ptr(),
                               table.data_ptr(), old.data_ptr(), 1, batch, rows, max_new, 0, 0)
                call = B.load().chiron_op_row_attention if fmt == "bf16" else B.load().chiron_op_row_attention8
                assert call(c.pool._h, 0, C.addressof(a), work.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
                torch.cuda.synchronize()
                assert (work[need:] == 0x5A).all() and (out[:rows] == 7.5).all() and (out[2 * rows:] == 7.5).all()
                got = out[rows:2 * rows].float()
                assert ((got == 7.5) | ((got - 1).abs() < 1e-2)).all()


@pytest.mark.parametrize("kw", (dict(max_new=1), dict(max_new=3), dict(max_new=20), dict(spare_rows=9), dict(layer=1, layers=3), dict(stride=8), dict(hot=30.0)))
def test_row_arguments(kw):
    for fmt, dtype in (("bf16", torch.float32), ("int8", torch.bfloat16)):
        check_rows(8, 2, 64, [50, 0, 20], [2, 40, 5], fmt, dtype, window=30, sinks=2, seed=11, **kw)
        check_rows(8, 2, 128, [50, 0, 20], [2, 1, 1], fmt, dtype, seed=12, **kw)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("new", (3, 24))
def test_not_finite_reaches_only_rows_that_see_it(dtype, new):
    """NaN and infinities in keys, values and queries of some tokens of a block of new ones, and of one that a window has passed"""
    n_q, n_kv, d, old, window = 4, 2, 64, 37, 20
    rng = np.random.default_rng(9)
    bt, blocks = L.tables([old + new], 3)
    c = L.Cache(n_kv, d, blocks, "bf16")
    c.fill(bt, [old + new], rng)
    k, v = c.pool.layer_views(0)
    k, v = (t.permute(0, 1, 2, 3, 4) if t.dim() == 5 else t for t in (k, v))
    q = torch.from_numpy(rng.standard_normal((new, n_q, d))).to(dtype).cuda()
    args = (L.dev(bt), ints([0, new]), ints([old]))
    clean = B.op_row_attention(c.pool, 0, q, *args, window=window).cpu()
    mid = new // 2
    bad = ((old + mid, 1, 5, float("nan")), (old + new - 1, 0, 9, float("inf")), (old - window + mid, 0, 33, float("-inf")))
    for p, h, e, x in bad:
        v[bt[0, p // PAGE], p % PAGE // 4, p % 4, h, e // 32, e % 32 // 16, e % 16] = x
    got = B.op_row_attention(c.pool, 0, q, *args, window=window).cpu()
    for r in range(new):
        for a in range(n_q):
            hit = {e for p, h, e, _ in bad if h == a // 2 and old + r - window < p <= old + r}
            for e in range(d):
                if e in hit:
                    assert not torch.isfinite(got[r, a, e]), (r, a, e)
                else:
                    assert got[r, a, e] == clean[r, a, e], (r, a, e)
    c.fill(bt, [old + new], np.random.default_rng(9))
    p = old + mid
    k[bt[0, p // PAGE], p % PAGE, 1, 0, 3] = float("nan")
    q[new - 1, 0, 7] = float("inf")
    got = B.op_row_attention(c.pool, 0, q, *args, window=window).cpu()
    for r in range(new):
        for a in range(n_q):
            if (a // 2 == 1 and r >= mid) or (a == 0 and r == new - 1):
                continue
            assert torch.equal(got[r, a], clean[r, a]), (r, a)


def test_row_attention_refusals():
    c = L.Cache(2, 64, 4, "int8")
    bt, starts, old = ints([[0, 1]]), ints([0, 2]), ints([3])
    q = torch.zeros((2, 4, 64), device="cuda")
    ok = dict(window=0, n_sinks=0)
    B.op_row_attention(c.pool, 0, q, bt, starts, old, **ok)
    for bad, err in (((c.pool, 1, q, bt, starts, old), B.ChironError), ((c.pool, 0, q.double(), bt, starts, old), TypeError),
                     ((c.pool, 0, q.cpu(), bt, starts, old), TypeError), ((c.pool, 0, q[:, :3].contiguous(), bt, starts, old), B.ChironError),
                     ((c.pool, 0, torch.zeros((2, 34, 64), device="cuda"), bt, starts, old), B.ChironError),
                     ((c.pool, 0, q, bt, starts[:1], old), ValueError), ((c.pool, 0, q, bt[0], starts, old), ValueError),
                     ((c.pool, 0, q, bt.long(), starts, old), TypeError), ((c.pool, 0, q.flatten(1), bt, starts, old), ValueError),
                     ((c.pool, 0, torch.zeros((2, 4 * 64 + 1), device="cuda")[:, :256].unflatten(1, (4, 64)), bt, starts, old), B.ChironError)):
        with pytest.raises(err):
            B.op_row_attention(*bad)
    for kw in (dict(window=-1), dict(n_sinks=-1), dict(max_new=-1)):
        with pytest.raises(B.ChironError):
            B.op_row_attention(c.pool, 0, q, bt, starts, old, **kw)
    with pytest.raises(ValueError):
        B.op_row_attention(c.pool, 0, q, bt, starts, old, out=q[:1])
    wide = torch.zeros((4, 4, 64), device="cuda")
    for out in (wide[:2], wide[1:3]):  # out over q, which other workgroups still read
        with pytest.raises(B.ChironError):
            B.op_row_attention(c.pool, 0, wide[:2], bt, starts, old, out=out)
    B.op_row_attention(c.pool, 0, wide[:2], bt, starts, old, out=wide[2:])
    with pytest.raises(B.ChironError):
        B.op_row_attention(c.pool, 0, q, bt[:0], ints([0]), old[:0])
    empty = q[:0]
    assert B.op_row_attention(c.pool, 0, empty, bt, ints([0, 0]), old).shape == empty.shape
    with pytest.raises(B.ChironError):
        B.KVPool8(c.model, 4, memory=torch.zeros(100, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.ChironError):
        B.KVPool8(c.model, 0)
