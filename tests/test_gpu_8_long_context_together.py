"""The long-context operators as an instance uses them, together: pages granted, rows rotated and appended, attended within a window, pages
released behind it; captured into a graph, on other streams, on pools beyond 4 GiB.  Needs a real MI355X: run with -m gpu.

Tolerances: attention as in test_gpu_7_long_context; everything else is equal (the operators take their sums in an order that follows
from the lengths alone)."""
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


def model(n_q, n_kv, d, width, layers=1):
    return B.Model(dict(n_layers=layers, hidden=16, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=d, ffn=16, vocab=16, rope_base=10000.0, rms_eps=1e-5), 1, width)


def pool_of(m, blocks, fmt):
    return B.KVPool(m, num_blocks=blocks) if fmt == "bf16" else B.KVPool8(m, blocks, fmt)


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
def test_an_instance_with_a_window(fmt):
    """six ticks of four requests: prompts, single tokens, rejected drafts, an ended request whose row a new one takes, pages behind the
    window given back; every tick's attention against 64 bits over what the cache holds, every page accounted for"""
    n_q, n_kv, d, width, blocks, window, sinks = 8, 2, 64, 12, 24, 40, 5
    G = n_q // n_kv
    m = model(n_q, n_kv, d, width)
    pool = pool_of(m, blocks, fmt)
    pages = B.PageList.of(blocks)
    bt = ints(np.full((4, width), -1))
    rng = np.random.default_rng(1)
    seen = [dict() for _ in range(4)]  # position -> (K, V) as the cache holds them
    old = np.zeros(4, np.int64)
    plan = ([70, 3, 0, 20], [1, 1, 50, 1], [4, 4, 4, 4], [1, 0, 1, 33], [90, 1, 2, 1], [1, 1, 1, 1])
    for step, new in enumerate(plan):
        if step == 3:  # two of the drafts of each request were rejected
            old -= 2
            pages.release(bt, ints(old))
        if step == 4:  # request 0 has ended, a prompt takes its row
            pages.release(bt, ints([0, 10 ** 6, 10 ** 6, 10 ** 6]))
            old[0], seen[0] = 0, {}
        total = sum(new)
        r = pages.grant(bt, ints(old), ints(new), total + 3)
        assert r.granted.tolist() == new and int(r.row_starts[-1]) == total
        x = torch.from_numpy(rng.standard_normal((total + 3, (n_q + 2 * n_kv) * d))).float().cuda()
        q, k, v = (t.unflatten(1, (-1, d)) for t in x.split((n_q * d, n_kv * d, n_kv * d), 1))
        cos, sin = B.rope_table(r.pos, d, 10000.0)
        out = torch.full((total + 3, n_q, d), 9.0, device="cuda")
        qr = pool.append_rope(0, k, v, cos, sin, bt, r.row_starts, ints(old), q=q)
        B.op_row_attention(pool, 0, qr, bt, r.row_starts, ints(old), window=window, n_sinks=sinks, max_new=max(new), out=out)
        torch.cuda.synchronize()
        say("tick", step, "old", old.tolist(), "new", new, "free", int(pages.count[0]))
        table = bt.cpu().numpy()
        assert sorted(table[table >= 0].tolist() + pages.pages[:int(pages.count[0])].tolist()) == list(range(blocks))
        slots = r.slots.cpu().numpy()
        for i in range(4):
            # the cache's own values: those of the pages that were written may have been rounded again
            first = int(old[i]) // PAGE * PAGE if new[i] else int(old[i])
            for p in range(first, int(old[i]) + new[i]):
                seen[i].pop(p, None)
            look = [p for p in range(first, int(old[i]) + new[i])]
            if look:
                if fmt == "bf16":
                    kk, vv = pool.gather(0, bt[i].contiguous(), int(old[i]) + new[i]) if (table[i, :-(-(int(old[i]) + new[i]) // PAGE)] >= 0).all() else (None, None)
                    for p in look:
                        if kk is not None:
                            seen[i][p] = (kk[p].double().cpu().numpy(), vv[p].double().cpu().numpy())
                        else:
                            a, b = pool.layer_views(0)
                            s = table[i, p // PAGE], p % PAGE
                            seen[i][p] = tuple(t.reshape(blocks, PAGE, n_kv, d)[s[0], s[1]].double().cpu().numpy() for t in (a, b))
                else:
                    kk, vv = pool.gather(0, bt, ints([i] * len(look)), ints(look))
                    for j, p in enumerate(look):
                        seen[i][p] = (kk[j].double().cpu().numpy(), vv[j].double().cpu().numpy())
            for t in range(new[i]):
                row, p = int(r.row_starts[i]) + t, int(old[i]) + t
                assert slots[row] == table[i, p // PAGE] * PAGE + p % PAGE
                see = [u for u in range(p + 1) if u > p - window or u < sinks]
                ks, vs = (np.stack([seen[i][u][j] for u in see]) for j in (0, 1))
                for h in range(n_kv):
                    want, slack = L.attend(qr[row, h * G:(h + 1) * G].double().cpu().numpy(), ks[:, h], vs[:, h], np.ones(len(see), bool))
                    tol = abs(vs).max() * (2 * slack + 2.0 ** -19 + 2 * (len(see) / 4 + 40) * 2.0 ** -24) + 2.0 ** -24 * abs(want)
                    assert (abs(out[row, h * G:(h + 1) * G].double().cpu().numpy() - want) <= tol).all(), (step, i, t, h)
        assert (out[total:] == 9.0).all()
        old += np.array(new)
        # what the windows have passed
        pages.release(bt, ints([sinks] * 4), ints(old - window + 1))


def workload(fmt, n_q=8, n_kv=2, d=64, batch=5, width=40, seed=3, rows_of=(1, 1, 1, 1, 1)):
    rng = np.random.default_rng(seed)
    m = model(n_q, n_kv, d, width)
    blocks = batch * width
    pool = pool_of(m, blocks, fmt)
    pool.memory.zero_()  # rows may see slots that nothing was appended to
    bt = ints(rng.permutation(blocks).reshape(batch, width))
    total = sum(rows_of)
    starts = ints(np.concatenate([[0], np.cumsum(rows_of)]))
    fill = [130, 0, 33, 500, 17][:batch]
    n = sum(fill)
    k, v = (torch.from_numpy(rng.standard_normal((n, n_kv, d))).float().cuda() for _ in range(2))
    pos = ints(np.concatenate([np.arange(f) for f in fill]))
    cos, sin = B.rope_table(pos, d, 10000.0)
    pool.append_rope(0, k, v, cos, sin, bt, ints(np.concatenate([[0], np.cumsum(fill)])), ints([0] * batch))
    return pool, bt, starts, np.array(fill), total, (n_q, n_kv, d), rng


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
@pytest.mark.parametrize("rows_of", ((1, 1, 1, 1, 1), (1, 60, 0, 2, 25)))
def test_captured_steps(fmt, rows_of):
    """append and attention in a graph, replayed with other rows and lengths, eager work and synchronizations in between: bit for bit what
    the eager calls give, and a second graph with a workspace of its own beside it"""
    pool, bt, starts, fill, total, (n_q, n_kv, d), rng = workload(fmt, rows_of=rows_of)
    twin, bt2 = pool_of(pool.model, 200, fmt), bt.clone()
    twin.memory.copy_(pool.memory)
    x = torch.zeros((total, (n_q + 2 * n_kv) * d), device="cuda")
    seq, cos, sin = ints(fill), torch.ones((total, d // 2), device="cuda"), torch.zeros((total, d // 2), device="cuda")

    def step(p, b):
        q, k, v = (t.unflatten(1, (-1, d)) for t in x.split((n_q * d, n_kv * d, n_kv * d), 1))
        qr = p.append_rope(0, k, v, cos, sin, b, starts, seq, q=q)
        return B.op_row_attention(p, 0, qr, b, starts, seq, window=70, n_sinks=3, max_new=max(rows_of)), B.op_row_attention(p, 0, qr.to(torch.bfloat16), b, starts, seq)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step(pool, bt)
    s.synchronize()
    torch.cuda.synchronize()
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(pool, bt)
    with torch.cuda.graph(g2):
        got2 = step(pool, bt)
    for t in range(4):
        x.copy_(torch.from_numpy(rng.standard_normal(x.shape)).float())
        pos = np.concatenate([np.arange(f + t, f + t + n) for f, n in zip(fill, rows_of)])
        c, sn = B.rope_table(ints(pos), d, 10000.0)
        cos.copy_(c)
        sin.copy_(sn)
        seq.copy_(ints(fill + t))
        torch.cuda.synchronize()
        (g if t % 2 == 0 else g2).replay()
        want = step(twin, bt2)
        torch.cuda.synchronize()
        for a, b in zip(got if t % 2 == 0 else got2, want):
            assert torch.equal(a, b)
        # (slots that nobody has written may hold anything in either pool)
        n = int(fill[0] + t + rows_of[0])
        if fmt == "bf16":
            assert torch.equal(pool.gather(0, bt[0].contiguous(), n)[0], twin.gather(0, bt2[0].contiguous(), n)[0])
        else:
            look = (ints([0] * n), ints(range(n)))
            assert torch.equal(pool.gather(0, bt, *look)[0], twin.gather(0, bt2, *look)[0])


def test_captured_tables():
    """grants and releases in a graph: the tables follow the lengths that the arrays hold at each replay"""
    rng = np.random.default_rng(8)
    for batch, width in ((6, 9), (1100, 3)):
        blocks = batch * 4
        pages, bt = B.PageList.of(blocks), ints(np.full((batch, width), -1))
        free, table = list(range(blocks)), np.full((batch, width), -1, np.int32)
        keep, new = ints([0] * batch), ints([1] * batch)

        def tick():
            pages.release(bt, keep)
            return pages.grant(bt, keep, new, 4 * batch)

        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            B.PageList.of(4).release(ints([[-1]]), ints([0]))
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m = tick()
        old = np.zeros(batch, np.int64)
        for t in range(4):
            n = rng.integers(0, 6, batch)
            keep.copy_(ints(old))
            new.copy_(ints(n))
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            free = L.release(table, free, old)
            free, starts, seq, pos, slots, granted = L.grant(table, free, old, n, 4 * batch)
            assert np.array_equal(bt.cpu().numpy(), table) and pages.pages[:int(pages.count[0])].tolist() == free
            for got, want in zip(m, (starts, seq, pos, slots, granted)):
                assert np.array_equal(got.cpu().numpy(), want)
            old += granted


def test_two_streams():
    """two calls at once, each with its own workspace and pool"""
    work = [workload(f, seed=s, rows_of=r) for f, s, r in (("int8", 1, (1, 1, 1, 1, 1)), ("bf16", 2, (1, 90, 0, 2, 25)))]
    ins = [torch.from_numpy(w[-1].standard_normal((w[4], w[5][0], w[5][2]))).float().cuda() for w in work]
    call = lambda i: B.op_row_attention(work[i][0], 0, ins[i], work[i][1], work[i][2], ints(work[i][3] - np.minimum(work[i][3], 20)), window=60, n_sinks=1)  # noqa: E731
    want = [call(0), call(1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for t in range(3):
        got = []
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                for _ in range(5):
                    out = call(i)
                got.append(out)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
def test_offsets_beyond_4_gib(fmt):
    """the same rows in a small pool and in the last pages of one beyond 4 GiB"""
    n_q, n_kv, d, width = 16, 8, 128, 12
    m = model(n_q, n_kv, d, width, layers=2)
    blocks = 45000 if fmt == "bf16" else 90000
    rng = np.random.default_rng(4)
    new = [100, 1, 60]
    total = sum(new)
    x = torch.from_numpy(rng.standard_normal((total, (n_q + 2 * n_kv) * d))).float().cuda()
    q, k, v = (t.unflatten(1, (-1, d)) for t in x.split((n_q * d, n_kv * d, n_kv * d), 1))
    starts = ints(np.concatenate([[0], np.cumsum(new)]))
    pos = np.concatenate([np.arange(n) for n in new])
    cos, sin = B.rope_table(ints(pos), d, 10000.0)
    ids = rng.permutation(3 * width).reshape(3, width)
    outs = []
    for nb, first in ((3 * width, 0), (blocks, blocks - 3 * width)):
        pool = pool_of(m, nb, fmt)
        assert nb < blocks or pool.memory.numel() > 1 << 32
        bt = ints(ids + first)
        qr = pool.append_rope(1, k, v, cos, sin, bt, starts, ints([0, 0, 0]), q=q)
        outs.append([B.op_row_attention(pool, 1, qr, bt, starts, ints([0, 0, 0]), window=50, n_sinks=2),
                     B.op_row_attention(pool, 1, qr[:3].contiguous(), bt, ints([0, 1, 2, 3]), ints([99, 0, 59]), max_new=1)])
        if fmt != "bf16":
            outs[-1] += list(pool.gather(1, bt, ints([0] * 100), ints(range(100))))
        torch.cuda.synchronize()
        say(fmt, "pages", nb, "bytes", pool.memory.numel())
        del pool
    torch.cuda.empty_cache()
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", ("bf16", "int8"))
def test_a_very_long_request(fmt):
    """one request of 300000 tokens in fp32, single tokens and a few, all of it and a window near its end, against 64 bits on the GPU"""
    n_q, n_kv, d, n = 4, 1, 64, 300000
    width = -(-n // PAGE) + 1
    m = model(n_q, n_kv, d, width)
    rng = np.random.default_rng(5)
    pool = pool_of(m, width, fmt)
    bt = ints(rng.permutation(width)[None])
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((n, n_kv, d), generator=g, device="cuda") for _ in range(2))
    one, zero = torch.ones((n, d // 2), device="cuda"), torch.zeros((n, d // 2), device="cuda")
    pool.append_rope(0, k, v, one, zero, bt, ints([0, n]), ints([0]))
    if fmt == "bf16":
        kk, vv = (t[:, 0].double() for t in pool.gather(0, bt[0].contiguous(), n))
    else:
        kk, vv = (t[:, 0].double() for t in pool.gather(0, bt, ints([0] * n), ints(range(n))))
    for new in (1, 3, 40):
        q = torch.randn((new, n_q, d), generator=g, device="cuda")
        for window, sinks in ((0, 0), (70001, 1000)):
            got = B.op_row_attention(pool, 0, q, bt, ints([0, new]), ints([n - new]), window=window, n_sinks=sinks).double()
            for t in range(new):
                p = torch.arange(n, device="cuda")
                at = n - new + t
                see = p <= at
                if window:
                    see &= (p > at - window) | (p < sinks)
                x = q[t].double() @ kk.t() / d ** 0.5
                slack = (d + 8) * 2.0 ** -24 * float((q[t].double().abs() @ kk.abs().t()).max()) / d ** 0.5
                want = torch.softmax(x.masked_fill(~see, -float("inf")), -1) @ vv
                # the sums' errors are those of their parts' sums: a share of a wave has at most a few thousand tokens, which lanes sum in fours
                tol = float(vv.abs().max()) * (2 * slack + 2.0 ** -19 + 2 * (n / 4 + 40) * 2.0 ** -24)
                assert float((got[t] - want).abs().max()) <= tol
                if new == 40 and t > 3:
                    break
