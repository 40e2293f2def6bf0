"""The drafting operators where they once went wrong, and loops of theirs that only larger calls reach: temperatures without end, row starts
out of order, small inputs beside large ones, zero points above 15, tables wider than the workspace, infinities in attended places.
Needs a real MI355X: run with -m gpu."""
import numpy as np
import pytest
import torch

import drafting as D
import test_gpu_4_drafting as T
import test_gpu_5_draft_and_verify as V
from paper_2501_08090_amd import binding as B
from paper_2501_08090_amd import drafting as DV
from paper_2501_08090_amd import inputs as I

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


def beside_large_ones(M, N, K, group, zeros, large, small, seed):
    """weights and x: one input of every 128 is `large` and meets weights of 0, the others are `small`"""
    w4, s, z = T.weights(N, K, group, zeros, seed)
    at = torch.arange(5, K, 128)
    zp = z[:, at // group] if zeros else torch.full((N, len(at)), 8, dtype=torch.uint8)
    w4[:, at // 2] = (w4[:, at // 2] & 15) | zp << 4
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, K), generator=g) * small
    x[:, at] = large * (1 + torch.rand((M, len(at)), generator=g)) * torch.where(torch.rand((M, len(at)), generator=g) < 0.5, -1, 1)
    return w4, s, z, x


@pytest.mark.parametrize("M,N,K", ((1, 200, 1024), (4, 200, 1024), (8, 200, 1024), (16, 200, 1024), (33, 200, 1024), (64, 4001, 8576)))
@pytest.mark.parametrize("group,zeros", ((128, False), (64, True), (32, False)))
@pytest.mark.parametrize("large,small", ((1e3, 1.0), (1e3, 2.0 ** -16), (1e5, 1.0)))
def test_linear4_small_inputs_beside_large_ones(M, N, K, group, zeros, large, small):
    """tolerance: x off by 2^-22 of itself and 2^-30.9 of the largest of its 128, for each product, and fp32 sums over the groups, of
    which an input's four digits can be twice its size"""
    w4, s, z, x = beside_large_ones(M, N, K, group, zeros, large, small, 71)
    lin = B.Linear4(w4.cuda(), s.cuda(), None if z is None else z.cuda())
    print("linear4", N, K, "group", group, "rows", M, "beside", large, small, flush=True)
    pick = np.r_[0:40, N - 40:N]
    w, _ = D.weights4(w4[pick], s[pick], None if z is None else z[pick], group)
    got = lin(x.cuda())[:, pick].double().cpu().numpy()
    xd = x.double().numpy()
    top = np.abs(xd).reshape(M, K // 128, 128).max(2).repeat(128, 1)
    off = 2.0 ** -22 * abs(xd) + 2.0 ** -30.9 * top
    parts = abs(xd) @ abs(w).T
    tol = off @ abs(w).T + 2 * (K // group + 6) * 2.0 ** -24 * parts
    err = abs(got - xd @ w.T)
    assert (err <= tol).all(), (err / tol).max()
    # and with all of the error in one direction: no input may be lost beside the large one
    if small == 1.0:
        x[:, torch.arange(K) % 128 != 5] = 0.75 * 2.0 ** -14
        ones = torch.full_like(w4, 0x99)
        ones[:, torch.arange(5, K, 128) // 2] = 0x89
        lin = B.Linear4(ones.cuda(), torch.ones_like(s).cuda())
        want = 0.75 * 2.0 ** -14 * (K - K // 128)
        tol = 2.0 ** -30.9 * 2 * large * K + 2.0 ** -21 * want
        assert abs(lin(x.cuda()).double().cpu().numpy() - want).max() <= tol


@pytest.mark.parametrize("M", (1, 3, 7, 16))
@pytest.mark.parametrize("zeros", (False, True))
@pytest.mark.parametrize("large", (1.98437, 1.98438, -1.98437, -1.98438, 1.0, 1.9999999))
def test_linear4_hands_x_through(M, zeros, large):
    """a matrix that hands x through: off by 2^-30.9 of the largest of the 128, and two roundings of digits up to twice x"""
    w4 = torch.full((128, 64), 0x88, dtype=torch.uint8)
    for n in range(128):
        w4[n, n // 2] = 0x98 if n % 2 else 0x89
    s = torch.ones((128, 1), dtype=torch.bfloat16)
    lin = B.Linear4(w4.cuda(), s.cuda(), torch.full((128, 1), 8, dtype=torch.uint8, device="cuda") if zeros else None)
    g = torch.Generator().manual_seed(M)
    x = (torch.rand((M, 128), generator=g) * 2 - 1) * 2.0 ** torch.randint(-12, 0, (M, 128), generator=g)
    x[:, 77] = large
    x[:, 78] = -large
    got = lin(x.cuda()).double().cpu()
    err = (got - x.double()).abs()
    assert (err <= 2.0 ** -30.9 * abs(large) + 2.0 ** -22 * x.double().abs()).all(), err.max()


@pytest.mark.parametrize("M,N,K,group", ((1, 40, 256, 128), (6, 40, 256, 64), (16, 40, 256, 32), (40, 75, 640, 32), (64, 4001, 8448, 128), (64, 2507, 8480, 32)))
def test_linear4_zero_points_up_to_64(M, N, K, group):
    """formats that store the zero point less one reach 16"""
    w4, s, z = T.weights(N, K, group, True, 81)
    z[:, ::2] = 16
    z[::3, 1::2] = torch.randint(0, 65, z[::3, 1::2].shape, generator=torch.Generator().manual_seed(1), dtype=torch.uint8)
    z[0] = 64
    pick = np.r_[0:20, N - 20:N]
    w, sk = D.weights4(w4[pick], s[pick], z[pick], group)
    lin = B.Linear4(w4.cuda(), s.cuda(), z.cuda())
    T.check_linear4(T.some_columns(lin, pick), w, sk, torch.randn((M, K), generator=torch.Generator().manual_seed(2)), group)


@pytest.mark.parametrize("where", ((0, 0), (39, 1), (17, 0)))
def test_linear4_refuses_larger_zero_points(where):
    w4, s, z = T.weights(40, 256, 128, True, 82)
    z[where] = 65
    with pytest.raises(B.ChironError) as e:
        B.Linear4(w4.cuda(), s.cuda(), z.cuda())
    assert e.value.code == -1 and "zero point" in str(e.value)
    z[where] = 64
    B.Linear4(w4.cuda(), s.cuda(), z.cuda())


@pytest.mark.parametrize("heads,rows,cols", (((1, 1, 64), 64, 16384), ((2, 2, 64), 40, 30000), ((4, 1, 128), 63, 120001)))
@pytest.mark.parametrize("pass_seq", (True, False))
def test_select_pages_of_tables_wider_than_the_workspace(heads, rows, cols, pass_seq):
    """rows x KV heads x columns beyond what the model's workspace holds of scores at once"""
    lens = [(r * 97) % 700 if r % 9 else 0 for r in range(rows)]
    lens[rows // 2], lens[-1] = 9000, 5001
    c, bt = T.filled(*heads, lens, 91, cols=cols)
    assert rows * heads[1] * cols > (8192 + 2 * 64) * heads[0] * heads[2]
    q = torch.randn((rows, heads[0] * heads[2]), generator=torch.Generator().manual_seed(1)).cuda()
    seq = list(range(rows))
    if pass_seq:
        seq = [(r * 7 + 3) % rows for r in seq]
    T.check_select(c, bt, q, [lens[s] for s in seq], seq, 33, 1, 1, pass_seq=pass_seq)


@pytest.mark.parametrize("batch,n,with_draft", ((257, 127, True), (257, 127, False), (65535, 0, True)))
def test_verify_largest_calls(batch, n, with_draft):
    """65535 rows of statistics, 2 n + 1 a request, are the most that one call takes"""
    logits, draft, tokens, u, noise = T.drafts(batch, n, 5, 95)
    assert batch * (2 * n + 1) == 65535
    T.check_verify(logits, tokens, u, noise, draft if with_draft else None, strict=False)
    more = [torch.cat((t, t[:1])).cuda() for t in (logits, tokens, u, noise)]
    with pytest.raises(B.ChironError) as e:
        B.verify_drafts(*more)
    assert e.value.code == -3


@pytest.mark.parametrize("heads", ((2, 2, 64), (8, 2, 128), (32, 2, 64)))
def test_sparse_attention_infinities_in_attended_places(heads):
    """a key or query that is none leaves its own head's outputs undefined, a value its own dim's, and nothing else"""
    n_q, n_kv, d = heads
    G = n_q // n_kv
    lens = [150, 90, 100]
    for what in ("key", "value", "query"):
        for val in (float("inf"), float("-inf"), float("nan")):
            c, bt = T.filled(*heads, lens, 97, spread=False)
            q = torch.randn((3, n_q * d), generator=torch.Generator().manual_seed(2)).cuda()
            ctx = D.dev(np.array(lens, np.int32))
            pages = D.dev(np.tile(np.arange(10, dtype=np.int32), (3, n_kv, 1)))
            want = B.op_sparse_attention(c.model, c.pool, 0, q, D.dev(bt), ctx, pages).view(3, n_q, d).clone()
            k, v = c.pool.layer_views(0)  # [page, token, head, d/8, 8] and [page, 4, 4 (token), head, d/32, 2, 16]
            if what == "key":
                k[int(bt[1, 2]), 3, 1, 2, 5] = val
            elif what == "value":
                v[int(bt[1, 2]), 1, 2, 1, 1, 1, 7] = val
            else:
                q[1, G * d + 9] = val
            print(what, val, flush=True)
            got = B.op_sparse_attention(c.model, c.pool, 0, q, D.dev(bt), ctx, pages).view(3, n_q, d)
            same = torch.ones((3, n_q, d), dtype=torch.bool, device="cuda")
            if what == "key":
                same[1, G:] = False
            elif what == "value":
                same[1, G:, 32 + 16 + 7] = False
                assert not got[1, G:, 32 + 16 + 7].isfinite().any()
            else:
                same[1, G] = False
            assert torch.equal(got[same], want[same])


def lists_near(q, c, bt, ctx, seq, top):
    """page lists of odd lengths for every row and KV head: a stride through the row's pages, shuffled"""
    rng = np.random.default_rng(5)
    lists = np.full((len(ctx), c.n_kv, top), -1, np.int32)
    counts = np.zeros(len(ctx), np.int32)
    for r, n in enumerate(ctx):
        pages = -(-n // 16)
        counts[r] = min(pages, top - r % 7)
        for h in range(c.n_kv):
            lists[r, h, :counts[r]] = rng.permutation(pages)[:counts[r]]
    return lists, counts


@pytest.mark.parametrize("heads", ((2, 2, 64), (8, 2, 128)))
def test_select_pages_long_lists_in_one_launch(heads):
    """128 lists and more, of several rounds of 512 pages each: every wave scores more than once 64 pages"""
    lens = [9601, 27199, 8192, 12000, 16001, 10001]
    c, bt = T.filled(*heads, lens, 101)
    rows = 64
    seq = [r % 6 for r in range(rows)]
    ctx = [lens[s] - 37 * (r // 6) for r, s in enumerate(seq)]
    ctx[7], ctx[8] = 513 * 16, 1024 * 16 + 1
    seq[7], seq[8] = 1, 1
    q = torch.randn((rows, heads[0] * heads[2]), generator=torch.Generator().manual_seed(3)).cuda()
    assert rows * heads[1] >= 128
    for top in (45, 700):
        T.check_select(c, bt, q, ctx, seq, top, 1, 1)


@pytest.mark.parametrize("top", (600, 701, 1100))
def test_sparse_attention_lists_that_a_wave_fetches_in_pieces(top):
    """129 lists and more, so that no list is split, with more than 64 entries a wave"""
    lens = [17000, 11111]
    c, bt = T.filled(3, 3, 64, lens, 102, spread=False)
    rows = 48
    seq = [r % 2 for r in range(rows)]
    ctx = [lens[s] - 5 * r for r, s in enumerate(seq)]
    q = torch.randn((rows, 192), generator=torch.Generator().manual_seed(4)).cuda()
    lists, counts = lists_near(q, c, bt, ctx, seq, top)
    assert rows * 3 > 128
    T.check_attend(c, bt, q, ctx, seq, D.dev(lists), D.dev(counts))


@pytest.mark.parametrize("M", (5, 8))
@pytest.mark.parametrize("zeros", (False, True))
@pytest.mark.parametrize("N,K", ((8003, 2080), (12001, 4096), (28671, 3104)))
def test_linear4_several_chunks_and_tiles(M, zeros, N, K):
    """groups of 32 and 5 to 8 rows: a workgroup goes through more than one chunk of K for more than one tile"""
    w4, s, z = T.weights(N, K, 32, zeros, 103)
    lin = B.Linear4(w4.cuda(), s.cuda(), None if z is None else z.cuda())
    pick = np.r_[0:20, 16 * 256:16 * 256 + 32, N // 2:N // 2 + 20, N - 40:N]
    w, sk = D.weights4(w4[pick], s[pick], None if z is None else z[pick], 32)
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(M))
    T.check_linear4(T.some_columns(lin, pick), w, sk, x, 32)
    T.check_linear4(T.some_columns(lin, pick), w, sk, x, 32, torch.randn((M, len(pick)), generator=torch.Generator().manual_seed(1)), True)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("shift", (0, 1))
def test_append_queries_that_go_past_the_caches(dtype, shift):
    """195 MiB of rotated queries; products and sums of the rotation in fp32"""
    n_q, d, rows = 16, 128, 25000
    c = D.Cache(n_q, 1, d, 1600)
    g = torch.Generator(device="cuda").manual_seed(9)
    whole = torch.randn((rows, (n_q + 2) * d + shift), generator=g, device="cuda").to(dtype)[:, shift:]
    q, k, v = (t.unflatten(1, (-1, d)) for t in whole.split((n_q * d, d, d), 1))
    cos, sin = B.rope_table(torch.arange(rows, dtype=torch.int32, device="cuda"), d, 10000.0)
    bt = torch.randperm(1600, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()[None]
    got = c.pool.append_rope(0, k, v, cos, sin, bt, D.dev(np.array([0, rows], np.int32)), D.dev(np.zeros(1, np.int32)), q=q)
    a, b = q.double().chunk(2, -1)
    cd, sd = cos.double()[:, None], sin.double()[:, None]
    off = (a.abs() + b.abs()) * 2.0 ** -22
    assert ((got[..., :d // 2] - (a * cd - b * sd)).abs() <= off).all() and ((got[..., d // 2:] - (b * cd + a * sd)).abs() <= off).all()
    stored = c.pool.layer_views(0)[1].reshape(1600, 16, 1, d)[bt[0].long()].view(-1, 1, d)[:rows]
    assert torch.equal(stored, v.to(torch.bfloat16))


@pytest.mark.parametrize("temperature", (0.0, 0.8))
def test_rounds_of_a_model_without_logits_go_on(temperature):
    """logits that are all NaN: the new token is -1, what the next round is fed is a token all the same"""
    m = dict(I.TINY)
    w = I.make_weights(m, seed=7, device="cuda", std=0.02)
    w["final_norm"] = torch.full_like(w["final_norm"], float("nan"))
    d, bt, sl = V.setup(m, np.array([20, 5], np.int32), 40, w, 64, 4, 24, seed=7)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    tokens = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    for r in range(2):
        out, accepted, sl, tokens = DV.draft_and_verify(d, bt, sl, tokens, 2, torch.full((2,), temperature, device="cuda"), g)
        assert (out == -1).all() and (accepted == 0).all() and (tokens == 0).all() and sl.tolist() == [21 + r, 6 + r]
