"""Where the long-context operators once went wrong.  Needs a real MI355X: run with -m gpu."""
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


@pytest.mark.parametrize("fmt", ("int8", "e4m3"))
@pytest.mark.parametrize("dtype,new", ((torch.float32, 1), (torch.bfloat16, 1), (torch.float32, 33)))
def test_small_weights_of_values_that_are_zero(fmt, dtype, new):
    """One token of weight 1 and value 1 before four million of about 2^-27 whose values are 0, in pages whose power of two is the smallest there is: these
    are part of the divisor, 1/60th of it or more, though they add nothing.  16 requests of 33 rows over 8 KV heads are 256 tiles, whose pages are not dealt out.

    The large weight and the value 1 are exact.  A small weight is off by the slack of its score (72 2^-24 of |q| |k| / sqrt(d), twice), its exponential's 2^-20
    and, with bf16 queries, 2^-9; a lane adds a quarter of them, with as many roundings of 2^-24.  The first four tokens of a page, whose lanes hold the large
    weight, have weights of 2^-54, which change nothing.  Then 16 roundings, and out's own to bf16, half a step below 1.  (Tiles of bf16 rows show nothing of it: there all
    weights come to one fp32 sum, which holds the 1 and may be off by 2^-24 for each that it adds, more than a weight of 2^-27 is.)"""
    n_q, n_kv, d, batch, pages = 32, 8, 64, 16, 1 << 18
    c = L.Cache(n_kv, d, 5, fmt)
    c.pool.memory.zero_()
    key, value = torch.zeros((80, n_kv, d), device="cuda"), torch.zeros((80, n_kv, d), device="cuda")
    key[[t for t in range(80) if t % PAGE < 4 or t >= 32], :, 0] = -1.0
    key[0, :, 0], value[0] = 1.0, 1.0
    one, zero = torch.ones((80, d // 2), device="cuda"), torch.zeros((80, d // 2), device="cuda")
    c.pool.append_rope(0, key, value, one, zero, ints([[0, 1, 2, 3, 4]]), ints([0, 80]), ints([0]))
    assert (c.pool.layer_views(0)[2][1, :, 1] == L.MIN_EXP).all()
    table = ints(np.tile(np.r_[0, np.ones(pages - 1), 2, 3, 4], (batch, 1)))
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn((batch * new, n_q, d), generator=g, device="cuda")
    q[:, :, 0] = (26.5 + torch.rand((batch * new, n_q), generator=g, device="cuda")) * (8 * np.log(2))
    q = q.to(dtype)
    say("small weights", fmt, dtype, new)
    got = B.op_row_attention(c.pool, 0, q, table, ints(np.arange(batch + 1) * new), ints([pages * PAGE] * batch), max_new=new).double().cpu().numpy()
    x = q[:, :, 0].double().cpu().numpy() / 8
    small = 12 * pages * np.exp(-x)
    want = 1.0 / (1.0 + small)  # the other tokens' weights, 2^-53 and less, are some 2^-35 together
    rel = 2 * 72 * 2.0 ** -24 * x + 2.0 ** -20 + (pages * 4 + 40) * 2.0 ** -24 + (2.0 ** -9 if dtype == torch.bfloat16 else 0.0)
    tol = small * rel + 16 * 2.0 ** -24 + (2.0 ** -9 if dtype == torch.bfloat16 else 0.0)
    assert small.min() > 2 * tol.max()  # else nothing would show
    err = abs(got - want[:, :, None]).max(-1)
    say("   worst error %.3f of what is allowed" % float((err / tol).max()))
    assert (err <= tol).all()


@pytest.mark.parametrize("fmt", ("int8", "e4m3", "bf16"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("new,large", ((1, 2.0 ** 127 * 1.5), (3, 2.0 ** 127 * 1.5), (1, -2.0 ** 127 * 1.9), (3, 2.0 ** 126 * 1.99), (33, -2.0 ** 113), (33, 2.0 ** 113)))
@pytest.mark.parametrize("n_q,n_kv,d", ((4, 1, 128), (8, 8, 64), (16, 2, 64)))
def test_queries_near_the_largest_number(fmt, dtype, new, large, n_q, n_kv, d):
    """Keys of 1 to 7 times +-2^-100 make scores of thousands and more that are whole multiples of one step: one token has all the weight, and the
    output is its value, exactly."""
    c = L.Cache(n_kv, d, 4, fmt)
    c.pool.memory.zero_()
    n = 3 * PAGE + 3
    key = torch.zeros((n, n_kv, d), device="cuda")
    key[:, :, 5] = ((torch.arange(n, device="cuda") % 6) - 3.0)[:, None] * 2.0 ** -100
    key[11, :, 5], key[17, :, 5] = -7 * 2.0 ** -100, 7 * 2.0 ** -100
    value = (torch.arange(n * n_kv * d, device="cuda") % 15 - 7.0).view(n, n_kv, d)  # held exactly by all three
    one, zero = torch.ones((n, d // 2), device="cuda"), torch.zeros((n, d // 2), device="cuda")
    table = ints([[2, 0, 3, 1]])
    c.pool.append_rope(0, key, value, one, zero, table, ints([0, n]), ints([0]))
    q = torch.zeros((new, n_q, d), dtype=dtype, device="cuda")
    q[:, :, 5] = large
    say("large", fmt, dtype, new, large)
    got = B.op_row_attention(c.pool, 0, q, table, ints([0, new]), ints([18]), max_new=new)
    want = value[17 if large > 0 else 11].repeat_interleave(n_q // n_kv, 0)
    assert (got.float() == want).all()


@pytest.mark.parametrize("fmt", ("bf16", "int8", "e4m3"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("new,window,sinks", ((1, 0, 0), (3, 0, 0), (40, 0, 0), (1, 70001, 1001), (3, 70001, 1001), (40, 70001, 1001)))
def test_every_share_of_a_very_long_request(fmt, dtype, new, window, sinks):
    """One request of 300000 tokens whose values say where a token is, so that a part of the pages that is lost or counted twice, or an edge that is off by a
    token, shows: dims 0 .. 31 are 1 in one of 32 runs of tokens, the others in single tokens around the edges of what a row sees.

    All values and weights are at least 0, so errors are relative.  A weight: twice the slack s of a score, twice the exponential's 2^-20, and with bf16 queries
    2^-9 in either sum.  Sums: a part of the pages holds a sixteenth of them at most, so n/16 additions and the joins' 100, each off by 2^-23 even if it cuts, in
    numerator and divisor.  bf16 results 2^-8."""
    n_q, n_kv, d, n = 4, 1, 64, 300000
    run, old = n // 32 + 1, n - new
    c = L.Cache(n_kv, d, -(-n // PAGE), fmt)
    g = torch.Generator(device="cuda").manual_seed(7)
    table = torch.randperm(-(-n // PAGE), generator=g, device="cuda").to(torch.int32)[None].contiguous()
    key = torch.randn((n, n_kv, d), generator=g, device="cuda") * 0.5
    at = torch.arange(n, device="cuda")
    value = torch.zeros((n, n_kv, d), device="cuda")
    value[at, 0, at // run] = 1.0
    edge = at > n - 70
    if window:
        edge |= (abs(at - (old - window)) < 70) | (abs(at - sinks) < 20)
    value[at[edge], 0, 32 + at[edge] % 32] = 1.0
    one, zero = torch.ones((n, d // 2), device="cuda"), torch.zeros((n, d // 2), device="cuda")
    c.pool.append_rope(0, key, value, one, zero, table, ints([0, n]), ints([0]))
    k, v = (torch.from_numpy(a[:, :, 0]).cuda()[table[0].long()].reshape(-1, d)[:n] for a in c.values())
    assert torch.equal(v.float(), value[:, 0])
    q = (torch.randn((new, n_q, d), generator=g, device="cuda") * 1.5).to(dtype)
    say("long", fmt, dtype, new, window, sinks)
    got = B.op_row_attention(c.pool, 0, q, table, ints([0, new]), ints([old]), window=window, n_sinks=sinks).double()
    worst = 0.0
    for t in sorted({0, 1, 2, new // 2, new - 1} & set(range(new))):
        see = at <= old + t
        if window:
            see &= (at > old + t - window) | (at < sinks)
        qt = q[t].double()
        w = torch.softmax((qt @ k.t().contiguous() / d ** 0.5).masked_fill(~see, -float("inf")), -1)
        want = w @ v
        slack = (d + 8) * 2.0 ** -24 * float((qt.abs() @ k.abs().t().contiguous()).max()) / d ** 0.5
        bf16 = dtype == torch.bfloat16
        rel = 2 * slack + 2.0 ** -19 + 2 * (int(see.sum()) / 16 + 100) * 2.0 ** -23 + (2 * 2.0 ** -9 + 2.0 ** -8 if bf16 else 0.0)
        # what a wave takes at least, 8 pages, would show (with bf16 rows four times as much)
        lost = 512 if bf16 else 128
        part = w[:, n // 2 // lost * lost + lost:old // lost * lost].reshape(n_q, -1, lost).sum(-1)
        if window:
            part = part[:, -(window - 4 * lost) // lost:]
        assert float(part.min()) > 1.5 * rel * float(want[:, :32].max())
        err = (got[t] - want).abs()
        worst = max(worst, float((err / (rel * want + 2.0 ** -60)).max()))
        assert (err <= rel * want).all(), (t, float((err - rel * want).max()))
    say("   worst error %.3f of what is allowed" % worst)


@pytest.mark.parametrize("fmt", ("int8", "e4m3", "bf16"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("new", (1, 3, 33))
@pytest.mark.parametrize("sign", (1.0, -1.0))
@pytest.mark.parametrize("n_q,n_kv,d", ((4, 1, 128), (8, 8, 64), (16, 2, 64)))
def test_scores_as_large_as_they_may_be(fmt, dtype, new, sign, n_q, n_kv, d):
    """Scores of one sign up to 2^29.8 whose distances are some 2^20 and more: one token has all the weight, and the output is its value, exactly."""
    c = L.Cache(n_kv, d, 4, fmt)
    c.pool.memory.zero_()
    n = 3 * PAGE + 3
    key = torch.zeros((n, n_kv, d), device="cuda")
    key[:, :, 5] = (2.0 + (torch.arange(n, device="cuda") % 4))[:, None] * 2.0 ** -20
    key[11, :, 5], key[17, :, 5] = 2.0 ** -20, 7 * 2.0 ** -20
    value = (torch.arange(n * n_kv * d, device="cuda") % 15 - 7.0).view(n, n_kv, d)
    one, zero = torch.ones((n, d // 2), device="cuda"), torch.zeros((n, d // 2), device="cuda")
    table = ints([[2, 0, 3, 1]])
    c.pool.append_rope(0, key, value, one, zero, table, ints([0, n]), ints([0]))
    q = torch.zeros((new, n_q, d), dtype=dtype, device="cuda")
    q[:, :, 5] = sign * 2.0 ** 50
    say("scores", fmt, dtype, new, sign)
    got = B.op_row_attention(c.pool, 0, q, table, ints([0, new]), ints([18]), max_new=new)
    want = value[17 if sign > 0 else 11].repeat_interleave(n_q // n_kv, 0)
    assert (got.float() == want).all()
