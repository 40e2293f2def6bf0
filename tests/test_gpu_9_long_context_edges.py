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
