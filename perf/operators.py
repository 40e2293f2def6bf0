"""The operators of drafted decoding: what an instance calls between two steps of the whole model when it drafts tokens cheaply from
the same cache and verifies them.

  append   keys and values of new tokens rotated and written to their pages, and the queries rotated; with `index`, the page index that
           block selection reads is brought up to date on the way
  sparse   one layer's attention of new tokens over the cache pages that a cheap score selects for each of them
  verify   drafted tokens accepted or replaced against the target's probabilities, from given random numbers
  linear4  products of few rows with a matrix of 4-bit weights with a scale (and, in some, a zero point) for each group

`run` computes them in plain torch in 32 bits (`own` false) or by the framework's entry points (`own` true); `exact` in 64 bits.  The
page index is exact integer arithmetic, the same in any precision: per page and head, a bound from above and one from below of
each key dimension, as whole multiples (-127 .. 127) of a power of two.
"""
import math
import random

import torch

own = False

PAGE = 16
TOP = float(torch.finfo(torch.float32).max)
TOP16 = float(torch.finfo(torch.bfloat16).max)
DEV = "cuda"


def _heads(q, kv, d):
    return dict(n_q_heads=q, n_kv_heads=kv, head_dim=d)


def listed():
    eight, small = _heads(32, 8, 128), _heads(16, 2, 64)
    return [
        # one decode step of the benchmark's batch: 64 requests bring one token each, fp32 rows of a fused projection
        dict(name="append_b64", op="append", batch=64, rows=64, median=800, dtype="f32", index=False, **eight),
        # the prompts of 37 requests of very different lengths enter a layer, some behind a shared prefix
        dict(name="append_ragged_5003", op="append", batch=37, rows=5003, median=300, dtype="bf16", index=False, **eight),
        # chunked prefill of four long prompts on an instance that drafts: the page index is written with the pages
        dict(name="append_index_16k", op="append", batch=4, rows=16384, median=2000, dtype="f32", index=True, **eight),
        # one interactive user drafts over 8k tokens: latency
        dict(name="sparse_b1_8k", op="sparse", batch=1, tokens=1, lo=8000, hi=8192, top=64, **eight),
        # the long-document batch drafts one token each, 2048 of some 28k tokens attended
        dict(name="sparse_b32_long32k", op="sparse", batch=32, tokens=1, lo=24576, hi=32768, top=128, **eight),
        # other head geometry, several tokens of each request at once, lengths from zero on
        dict(name="sparse_b61x3_ragged", op="sparse", batch=61, tokens=3, lo=0, hi=5000, top=33, **small),
        # one user, four drafted tokens
        dict(name="verify_b1_n4", op="verify", batch=1, drafts=4, vocab=128256, with_draft=True),
        # the benchmark's batch, four drafted tokens each
        dict(name="verify_b64_n4", op="verify", batch=64, drafts=4, vocab=128256, with_draft=True),
        # drafts without probabilities (looked up in the text), ragged numbers of them, an odd vocabulary
        dict(name="verify_b23_n7_odd", op="verify", batch=23, drafts=7, vocab=50257, with_draft=False),
        # one row through a square matrix: the smallest projection of a draft step
        dict(name="linear4_r1_4096", op="linear4", rows=1, n=4096, k=4096, group=128, zeros=False),
        # eight requests through the fused gate and up matrix of the 8B shape
        dict(name="linear4_r8_gateup", op="linear4", rows=8, n=28672, k=4096, group=128, zeros=False),
        # 64 requests through the down matrix of the 70B shape, finer groups with zero points
        dict(name="linear4_r64_down70b", op="linear4", rows=64, n=8192, k=28672, group=64, zeros=True),
    ]


def _log(rng, lo, hi):
    """a whole number, spread evenly over the logarithm of the range"""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "sparse", "verify", "linear4"))
    if op in ("append", "sparse"):
        kv = rng.choice((1, 2, 4, 8))
        heads = _heads(kv * rng.choice((1, 2, 4, 8, 16) if kv < 8 else (1, 2, 4, 8)), kv, rng.choice((64, 128)))
    if op == "append":
        rows = _log(rng, 1, 16384)
        return dict(op=op, batch=rng.randint(1, min(rows, 64)), rows=rows, median=_log(rng, 16, 2000), dtype=rng.choice(("f32", "bf16")),
                    index=rows >= 2048 and rng.random() < 0.5, **heads)
    if op == "sparse":
        hi = _log(rng, 16, 32768)
        batch = _log(rng, 1, min(64, max(1, 900000 // hi)))
        return dict(op=op, batch=batch, tokens=rng.choice((1, 1, 2, 3, 5)) if hi < 8192 else 1, lo=rng.choice((0, hi // 2)), hi=hi,
                    top=_log(rng, 3, 128), **heads)
    if op == "verify":
        drafts = _log(rng, 1, 8)
        return dict(op=op, batch=_log(rng, 1, 256 // (drafts + 1)), drafts=drafts, vocab=_log(rng, 1000, 128256), with_draft=rng.random() < 0.7)
    group = rng.choice((32, 64, 128))
    return dict(op=op, rows=_log(rng, 1, 64), n=_log(rng, 500, 28672), k=group * _log(rng, 512 // group, 14336 // group), group=group,
                zeros=rng.random() < 0.5)


# ---- inputs, made from the seed alone --------------------------------------------------------------------------

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + salt) & 0x7FFFFFFFFFFF)
    return g


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _tables(lens, seed):
    """distinct pages in random order for each request, -1 where it has none, and the number of pages of the pool"""
    need = [-(-max(1, n) // PAGE) for n in lens]
    total = sum(need)
    blocks = total + total // 8 + 1
    ids = torch.randperm(blocks, generator=torch.Generator().manual_seed(seed + 17))[:total].tolist()
    bt, o = [], 0
    for n in need:
        bt.append(ids[o:o + n] + [-1] * (max(need) - n))
        o += n
    return _i32(bt), blocks


def _pool(c, blocks, rows, width):
    """the framework's pool for one layer of these heads: the handles that a program keeps"""
    from paper_2501_08090_amd import binding as B
    m = dict(n_layers=1, hidden=16, ffn=16, vocab=16, rope_base=10000.0, rms_eps=1e-5, **{k: c[k] for k in ("n_q_heads", "n_kv_heads", "head_dim")})
    model = B.Model(m, rows, width)
    return model, B.KVPool(model, num_blocks=blocks)


def _views(c, k, v):
    """a plain cache [pages, 16, heads, d] in the shapes of the pool's views"""
    nb, _, nkv, d = k.shape
    return k.view(nb, PAGE, nkv, d // 8, 8), v.view(nb, 4, 4, nkv, d // 32, 2, 16)


def _cache(c, blocks, seed):
    """K and V of every page: keys of a page resemble each other, as neighbouring tokens' do"""
    g = _gen(seed, 1)
    shape = (blocks, PAGE, c["n_kv_heads"], c["head_dim"])
    k = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    k.mul_(0.8).add_(torch.randn((blocks, 1) + shape[2:], generator=g, device=DEV, dtype=torch.bfloat16), alpha=0.6)
    return k, torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)


def _prepare_append(c, seed):
    r = random.Random(17)  # the lengths are the case's own, in an order that goes by the seed
    B_, rows, d, nq, nkv = c["batch"], c["rows"], c["head_dim"], c["n_q_heads"], c["n_kv_heads"]
    share = [math.exp(r.gauss(0, 1.5)) if rows > B_ else 1.0 for _ in range(B_)]
    new = [1 + int((rows - B_) * s / sum(share)) for s in share]
    new[0] += rows - sum(new)
    old = [min(4096, int(c["median"] * math.exp(r.gauss(0, 0.8)))) if r.random() < 0.8 else 0 for _ in range(B_)]
    order = random.Random(seed).sample(range(B_), B_)
    old, new = [old[i] for i in order], [new[i] for i in order]
    bt, blocks = _tables([a + b for a, b in zip(old, new)], seed)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    g = _gen(seed, 2)
    width = (nq + 2 * nkv) * d
    qkv = torch.randn((rows, width), generator=g, device=DEV, dtype=torch.float32)
    if c["dtype"] == "bf16":
        qkv = qkv.to(torch.bfloat16)
    s = dict(case=c, qkv=qkv, q=qkv[:, :nq * d].unflatten(1, (nq, d)), k=qkv[:, nq * d:(nq + nkv) * d].unflatten(1, (nkv, d)),
             v=qkv[:, (nq + nkv) * d:].unflatten(1, (nkv, d)), block_table=bt, row_starts=_i32(starts), seq_lens=_i32(old))
    pos = torch.cat([torch.arange(o, o + n) for o, n in zip(old, new)]).to(DEV)
    angle = pos.double()[:, None] * 500000.0 ** (-2.0 * torch.arange(d // 2, device=DEV).double() / d)
    s["angle"] = angle
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    k, v = _cache(c, blocks, seed)
    s["K"], s["V"] = k, v
    if c["index"]:
        s["codes"] = torch.zeros((blocks, nkv, 2, d), dtype=torch.int8, device=DEV)
        s["exps"] = torch.zeros((blocks, nkv), dtype=torch.int8, device=DEV)
    return s, blocks


def _prepare_sparse(c, seed):
    r = random.Random(19)
    B_, t, d, nq, nkv = c["batch"], c["tokens"], c["head_dim"], c["n_q_heads"], c["n_kv_heads"]
    lens = [r.randint(c["lo"], c["hi"]) for _ in range(B_)]  # tokens that the last new token of each request sees
    if B_ > 8 and c["lo"] == 0:
        lens[1], lens[2] = 0, 1
    random.Random(seed).shuffle(lens)
    bt, blocks = _tables(lens, seed)
    ctx = [max(0, n - t + 1 + j) if n else 0 for n in lens for j in range(t)]
    g = _gen(seed, 2)
    s = dict(case=c, q=torch.randn((B_ * t, nq * d), generator=g, device=DEV, dtype=torch.float32) * 1.5, block_table=bt, ctx_lens=_i32(ctx),
             row_seq=_i32([i for i in range(B_) for _ in range(t)]))
    s["K"], s["V"] = _cache(c, blocks, seed)
    valid = torch.full((blocks,), PAGE, dtype=torch.int64, device=DEV)
    for i, n in enumerate(lens):
        if n % PAGE:
            valid[bt[i, n // PAGE].long()] = n % PAGE
    parts = [_index(s["K"][i:i + 4096], valid[i:i + 4096]) for i in range(0, blocks, 4096)]
    s["codes"], s["exps"] = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
    return s, blocks


def _own_cache(s, c, blocks, rows):
    """the same cache in the framework's pool, and its page index"""
    from paper_2501_08090_amd import binding as B
    s["model"], s["pool"] = _pool(c, blocks, rows, s["block_table"].shape[1])
    k, v = s["pool"].layer_views(0)
    a, b = _views(c, s.pop("K"), s.pop("V"))
    k.copy_(a)
    v.copy_(b)
    if "codes" in s:
        s["index"] = B.KVIndex(s["pool"])
        codes, exps = s["index"].layer_views(0)
        codes.copy_(s.pop("codes"))
        exps.copy_(s.pop("exps"))


def _prepare_verify(c, seed):
    r = random.Random(seed * 7 + 5)
    B_, n, V = c["batch"], c["drafts"], c["vocab"]
    g = _gen(seed, 3)
    # logits of a model that is sure of some tokens and not of others, and of a draft that mostly agrees with it
    logits = torch.randn((B_, n + 1, V), generator=g, device=DEV, dtype=torch.float32) * 2.5
    sharp = torch.rand((B_, n + 1, 1), generator=g, device=DEV) * 2.0
    logits *= sharp
    s = dict(case=c, logits=logits, noise=torch.empty((B_, V), device=DEV).exponential_(generator=g),
             uniforms=torch.rand((B_, n), generator=g, device=DEV))
    T = [0.0 if r.random() < 0.2 else 0.5 + r.random() for _ in range(B_)]
    T[0] = 0.8
    s["temperature"] = torch.tensor(T, dtype=torch.float32, device=DEV)
    s["draft_lens"] = _i32([n if B_ == 1 or r.random() < 0.7 else r.randint(0, n) for _ in range(B_)])
    s["draft_logits"] = None
    near = logits[:, :n] + 0.5 * torch.randn((B_, n, V), generator=g, device=DEV)
    soft = torch.softmax(near / s["temperature"].clamp(min=0.05)[:, None, None], -1).view(B_ * n, V)
    s["tokens"] = torch.multinomial(soft, 1, generator=g).view(B_, n).to(torch.int32)
    if c["with_draft"]:
        s["draft_logits"] = near
    return s


def _prepare_linear4(c, seed):
    g = _gen(seed, 4)
    N, K, G = c["n"], c["k"], c["group"]
    s = dict(case=c, w4=torch.randint(0, 256, (N, K // 2), generator=g, device=DEV, dtype=torch.uint8),
             scales=(0.002 + 0.008 * torch.rand((N, K // G), generator=g, device=DEV)).to(torch.bfloat16), zeros=None)
    if c["zeros"]:
        s["zeros"] = torch.randint(5, 11, (N, K // G), generator=g, device=DEV, dtype=torch.uint8)
    x = torch.randn((c["rows"], K), generator=g, device=DEV)
    # a few channels are much larger than the others, as in a decoder's residual stream
    x[:, torch.randperm(K, generator=torch.Generator().manual_seed(seed))[:max(1, K // 256)].to(DEV)] *= 20.0
    s["x"] = x
    return s


def prepare(case, seed):
    op = case["op"]
    if op == "append" or op == "sparse":
        s, blocks = (_prepare_append if op == "append" else _prepare_sparse)(case, seed)
        s.pop("angle", None)
        if own:
            _own_cache(s, case, blocks, case["batch"] * case.get("tokens", 1))
        return s
    if op == "verify":
        return _prepare_verify(case, seed)
    s = _prepare_linear4(case, seed)
    if own:
        from paper_2501_08090_amd import binding as B
        s["linear"] = B.Linear4(s.pop("w4"), s.pop("scales"), s.pop("zeros"))
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------

def _power(amax):
    """the exponent e of the smallest power of two with amax <= 127 * 2^e, at least -126"""
    mant, ex = torch.frexp(amax)
    e = ex - 7 + (mant > 127.0 / 128.0)
    return torch.where(amax > 0, e, torch.zeros_like(e)).clamp(min=-126)


def _two(e):
    """2^e as an exact fp32 value, -126 <= e <= 127"""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _finite(x, top):
    return torch.where(torch.isnan(x), torch.zeros_like(x), x).clamp(-top, top)


def _index(k, valid):
    """codes [n, heads, 2, d] (from above, from below) and exponents [n, heads] of pages k [n, 16, heads, d] with `valid` tokens each"""
    x = _finite(k.float(), TOP16)
    there = (torch.arange(PAGE, device=DEV)[None, :] < valid[:, None])[:, :, None, None]
    hi = torch.where(there, x, torch.full_like(x, -math.inf)).amax(1)
    lo = torch.where(there, x, torch.full_like(x, math.inf)).amin(1)
    e = _power(torch.maximum(hi.abs(), lo.abs()).amax(-1))
    up = _two(-e)[..., None]
    return torch.stack((torch.ceil(hi * up), torch.floor(lo * up)), 2).to(torch.int8), e.to(torch.int8)


def _rotate(x, cos, sin):
    """pairs (j, j + d/2) of x [rows, heads, d] turned by their row's angles"""
    x = x.float()
    a, b = x.chunk(2, -1)
    c, s = cos[:, None, :], sin[:, None, :]
    return torch.cat((a * c - b * s, b * c + a * s), -1)


def _places(s):
    """page and slot of each new row"""
    rows = s["q"].shape[0]
    row = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(s["row_starts"].long(), row, right=True) - 1
    pos = s["seq_lens"].long()[seq] + row - s["row_starts"].long()[seq]
    return row, seq, pos, s["block_table"].long()[seq, pos // PAGE]


def _append_plain(s):
    row, seq, pos, page = _places(s)
    s["K"][page, pos % PAGE] = _rotate(s["k"], s["cos"], s["sin"]).to(torch.bfloat16)
    s["V"][page, pos % PAGE] = s["v"].to(torch.bfloat16)
    out = dict(q=_rotate(s["q"], s["cos"], s["sin"]))
    out["k"], out["v"] = _views(s["case"], s["K"], s["V"])
    if "codes" in s:
        first = (pos % PAGE == 0) | (row == s["row_starts"].long()[seq])
        end = (s["seq_lens"].long() + s["row_starts"].long()[1:] - s["row_starts"].long()[:-1])[seq]
        p = page[first]
        valid = (end - pos // PAGE * PAGE).clamp(max=PAGE)[first]
        s["codes"][p], s["exps"][p] = _index(s["K"][p], valid)
        out["bounds"] = s["codes"] * _two(s["exps"])[:, :, None, None]
    return out


def _select_plain(s):
    c = s["case"]
    top, d, nkv = c["top"], c["head_dim"], c["n_kv_heads"]
    rows = s["q"].shape[0]
    q = _finite(s["q"], TOP).view(rows, nkv, -1, d)
    e = _power(q.abs().amax((2, 3)))
    q8 = torch.round(q * _two(-e)[:, :, None, None])
    bt = s["block_table"].long()[s["row_seq"].long()]
    P = bt.shape[1]
    phys = bt.clamp(min=0)
    codes = s["codes"][phys].permute(0, 2, 1, 3, 4).reshape(rows, nkv, P, 2 * d).float()
    q2 = torch.cat((q8.clamp(min=0), q8.clamp(max=0)), -1)
    score = torch.matmul(codes, q2.transpose(2, 3)).amax(-1)
    score = (score * _two(s["exps"][phys].permute(0, 2, 1))).clamp(-TOP, TOP)
    n = ((s["ctx_lens"].long() + PAGE - 1) // PAGE)[:, None, None]
    page = torch.arange(P, device=DEV)[None, None, :]
    score = torch.where((page < 1) | (page == n - 1), torch.full_like(score, math.inf), score)
    score = torch.where(page < n, score, torch.full_like(score, -math.inf))
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :top]
    if P < top:
        order = torch.nn.functional.pad(order, (0, top - P), value=P)
    count = n.clamp(max=top)
    order = torch.where(torch.arange(top, device=DEV) < count, order, torch.full_like(order, 1 << 40)).sort(-1).values
    return torch.where(order < (1 << 40), order, torch.full_like(order, -1)).to(torch.int32), count.view(rows).to(torch.int32)


def _attend_plain(s, pages):
    c = s["case"]
    d, nkv = c["head_dim"], c["n_kv_heads"]
    rows = s["q"].shape[0]
    q = s["q"].view(rows, nkv, -1, d)
    bt = s["block_table"].long()[s["row_seq"].long()]
    there = pages >= 0
    logical = pages.long().clamp(min=0)
    phys = torch.gather(bt[:, None, :].expand(rows, nkv, bt.shape[1]), 2, logical).clamp(min=0)
    head = torch.arange(nkv, device=DEV)[None, :, None]
    top = pages.shape[2]
    k = s["K"].permute(0, 2, 1, 3)[phys, head].reshape(rows, nkv, top * PAGE, d)
    v = s["V"].permute(0, 2, 1, 3)[phys, head].reshape(rows, nkv, top * PAGE, d)
    tok = logical[..., None] * PAGE + torch.arange(PAGE, device=DEV)
    live = (there[..., None] & (tok < s["ctx_lens"].long()[:, None, None, None])).reshape(rows, nkv, 1, top * PAGE)
    x = torch.matmul(q, k.float().transpose(2, 3)) / math.sqrt(d)
    x = torch.where(live, x, torch.full_like(x, -math.inf))
    m = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    z = w.sum(-1, keepdim=True)
    vf = torch.where(live.transpose(2, 3), v.float(), torch.zeros((), device=DEV))
    out = torch.matmul(w, vf) / torch.where(z > 0, z, torch.ones_like(z))
    return out.reshape(rows, -1)


def _shares(z, T):
    """softmax of z / T over the last dimension; zeros where nothing is left"""
    z = torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z).clamp(max=TOP)
    m = z.amax(-1, keepdim=True)
    w = torch.exp((z - torch.where(torch.isinf(m), torch.zeros_like(m), m)) * (1.0 / T))
    return w / w.sum(-1, keepdim=True).clamp(min=1e-38)


def _verify_plain(s):
    B_, n1, V = s["logits"].shape
    n = n1 - 1
    T = s["temperature"]
    greedy = T == 0
    T1 = torch.where(greedy, torch.ones_like(T), T)[:, None, None]
    tok = s["tokens"].long()
    best = s["logits"].argmax(-1)
    p = _shares(s["logits"], T1)
    px = torch.gather(p[:, :n], 2, tok[..., None]).squeeze(-1)
    if s["draft_logits"] is not None:
        q = _shares(s["draft_logits"], T1)
        qx = torch.gather(q, 2, tok[..., None]).squeeze(-1)
    else:
        q, qx = None, torch.ones_like(px)
    prob = torch.where(qx > 0, px / qx, (px > 0).float()).clamp(max=1.0)
    prob = torch.where(greedy[:, None], (tok == best[:, :n]).float(), prob)
    at = torch.arange(n, device=DEV)
    lens = s["draft_lens"].long()
    prob = torch.where(at[None, :] < lens[:, None], prob, torch.zeros_like(prob))
    took = torch.cumprod((s["uniforms"] < prob).long(), 1).sum(1)
    b = torch.arange(B_, device=DEV)
    full = p[b, took]
    left = full
    if n:
        j = took.clamp(max=n - 1)
        if q is not None:
            rest = (full - q[b, j]).clamp(min=0)
        else:
            rest = full.clone()
            rest[b, tok[b, j]] = 0
        use = (took < lens) & (rest.amax(-1) > 0)
        left = torch.where(use[:, None], rest, full)
    race = torch.where(left > 0, left / s["noise"], torch.full_like(left, -1.0))
    new = torch.where(greedy, best[b, took], race.argmax(-1))
    out = torch.where(torch.arange(n1, device=DEV)[None, :] < took[:, None], torch.nn.functional.pad(tok, (0, 1)), torch.full_like(best, -1))
    out[b, took] = new
    return dict(tokens=out.to(torch.int32), accepted=took.to(torch.int32), prob=prob)


def _linear4_plain(s):
    c = s["case"]
    N, K, G = c["n"], c["k"], c["group"]
    w4 = s["w4"]
    q = torch.stack((w4 & 15, w4 >> 4), -1).view(N, K // G, G).float()
    z = s["zeros"].float()[..., None] if s["zeros"] is not None else 8.0
    w = ((q - z) * s["scales"].float()[..., None]).view(N, K)
    return torch.matmul(s["x"], w.t())


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "append":
            return _append_plain(s)
        if op == "sparse":
            pages, counts = _select_plain(s)
            return dict(pages=pages, counts=counts, out=_attend_plain(s, pages))
        return _verify_plain(s) if op == "verify" else dict(y=_linear4_plain(s))
    from paper_2501_08090_amd import binding as B
    if op == "append":
        out = dict(q=s["pool"].append_rope(0, s["k"], s["v"], s["cos"], s["sin"], s["block_table"], s["row_starts"], s["seq_lens"], q=s["q"],
                                           index=s.get("index")))
        out["k"], out["v"] = s["pool"].layer_views(0)
        if "index" in s:
            codes, exps = s["index"].layer_views(0)
            out["bounds"] = codes * _two(exps)[:, :, None, None]
        return out
    if op == "sparse":
        pages, counts = B.op_select_pages(s["model"], s["pool"], s["index"], 0, s["q"], s["block_table"], s["ctx_lens"], s["case"]["top"],
                                          n_first=1, n_last=1, row_seq=s["row_seq"])
        out = B.op_sparse_attention(s["model"], s["pool"], 0, s["q"], s["block_table"], s["ctx_lens"], pages, counts, row_seq=s["row_seq"])
        return dict(pages=pages, counts=counts, out=out)
    if op == "verify":
        tokens, accepted, prob = B.verify_drafts(s["logits"], s["tokens"], s["uniforms"], s["noise"], draft_logits=s["draft_logits"],
                                                 draft_lens=s["draft_lens"], temperature=s["temperature"])
        return dict(tokens=tokens, accepted=accepted, prob=prob)
    return dict(y=s["linear"](s["x"]))


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def work(c):
    op = c["op"]
    if op == "append":
        q, kv = c["n_q_heads"] * c["head_dim"], 2 * c["n_kv_heads"] * c["head_dim"]
        size = 4 if c["dtype"] == "f32" else 2
        # rows in; rotated queries, keys and values out; the rotary table; the index of the pages that are written
        per_row = (q + kv) * size + 4 * q + 2 * kv + 4 * c["head_dim"]
        return dict(bytes=c["rows"] * per_row + (c["rows"] // PAGE * c["n_kv_heads"] * (2 * c["head_dim"] + 1) if c["index"] else 0),
                    flops=3 * c["rows"] * (q + kv // 2))
    if op == "sparse":
        rows, n = c["batch"] * c["tokens"], (c["lo"] + c["hi"]) / 2
        pages = -(-n // PAGE)
        d, nq, nkv = c["head_dim"], c["n_q_heads"], c["n_kv_heads"]
        took = min(pages, c["top"])
        # the index of a request's pages once, the selected pages of each row, rows in and out, the lists
        return dict(bytes=c["batch"] * pages * nkv * (2 * d + 1) + rows * nkv * took * PAGE * d * 4 + rows * nq * d * 8 + rows * nkv * c["top"] * 4,
                    flops=rows * nq * (pages * 4 * d + took * PAGE * 4 * d))
    if op == "verify":
        B_, n, V = c["batch"], c["drafts"], c["vocab"]
        return dict(bytes=4 * V * B_ * (n + 1 + (n if c["with_draft"] else 0) + 1), flops=4 * V * B_ * (2 * n + 2))
    M, N, K, G = c["rows"], c["n"], c["k"], c["group"]
    return dict(bytes=N * K // 2 + N * (K // G) * (3 if c["zeros"] else 2) + 4 * M * (N + K), flops=2 * M * N * K)


# ---- the same in 64 bits, written apart ------------------------------------------------------------------------

def _exact_append(c, seed):
    s, blocks = _prepare_append(c, seed)
    K, V = s["K"].double(), s["V"].double()
    starts, old, bt = s["row_starts"].tolist(), s["seq_lens"].tolist(), s["block_table"].tolist()
    half = c["head_dim"] // 2
    cos, sin = s["cos"].double()[:, None], s["sin"].double()[:, None]

    def turned(x):
        x = x.double()
        y = torch.empty_like(x)
        y[..., :half] = x[..., :half] * cos - x[..., half:] * sin
        y[..., half:] = x[..., half:] * cos + x[..., :half] * sin
        return y

    k, v = turned(s["k"]), s["v"].double()
    for i in range(c["batch"]):
        for pg in range(old[i] // PAGE, (old[i] + starts[i + 1] - starts[i] - 1) // PAGE + 1):
            a, b = max(old[i], pg * PAGE), min(old[i] + starts[i + 1] - starts[i], pg * PAGE + PAGE)
            src = slice(starts[i] + a - old[i], starts[i] + b - old[i])
            K[bt[i][pg], a - pg * PAGE:b - pg * PAGE], V[bt[i][pg], a - pg * PAGE:b - pg * PAGE] = k[src], v[src]
    out = dict(q=turned(s["q"]), k=K, v=V)
    if c["index"]:
        out["bounds"] = None  # follows from the rounded keys, not from these
    return out


def _exact_sparse(c, seed):
    s, blocks = _prepare_sparse(c, seed)
    d, nkv, top = c["head_dim"], c["n_kv_heads"], c["top"]
    G = c["n_q_heads"] // nkv
    q = s["q"].double().view(-1, nkv, G, d)
    bt, ctx, seq = s["block_table"].long(), s["ctx_lens"].tolist(), s["row_seq"].tolist()
    out = torch.zeros_like(q)
    for r in range(q.shape[0]):
        n = -(-ctx[r] // PAGE)
        if n == 0:
            continue
        page = bt[seq[r], :n]
        codes, ex = s["codes"][page].double(), s["exps"][page].long()
        for h in range(nkv):
            x = q[r, h]
            mant, e = math.frexp(float(x.abs().max()))
            x8 = torch.round(x * 2.0 ** -max(-126, e - 7 + (mant > 127 / 128)))
            score = (torch.einsum("gd,pd->pg", x8.clamp(min=0), codes[:, h, 0]) + torch.einsum("gd,pd->pg", x8.clamp(max=0), codes[:, h, 1])).max(1).values
            score = score * ((ex[:, h] + 1023) << 52).view(torch.float64)
            score[0] = score[n - 1] = math.inf
            chosen = torch.sort(score, descending=True, stable=True).indices[:min(top, n)]
            k = s["K"][page[chosen], :, h].double().reshape(-1, d)
            v = s["V"][page[chosen], :, h].double().reshape(-1, d)
            live = ((chosen * PAGE)[:, None] + torch.arange(PAGE, device=DEV) < ctx[r]).reshape(-1)
            out[r, h] = torch.softmax((x @ k[live].t()) / math.sqrt(d), -1) @ v[live]
    return dict(pages=None, counts=None, out=out)


def _exact_verify(c, seed):
    s = _prepare_verify(c, seed)
    B_, n = c["batch"], c["drafts"]
    prob = torch.zeros((B_, n), dtype=torch.float64, device=DEV)
    T, lens, tok = s["temperature"].double().tolist(), s["draft_lens"].tolist(), s["tokens"].tolist()
    for i in range(B_):
        for t in range(lens[i]):
            x, z = tok[i][t], s["logits"][i, t].double()
            if T[i] == 0:
                prob[i, t] = float(int(z.argmax()) == x)
                continue
            lp = z[x] / T[i] - torch.logsumexp(z / T[i], 0)
            if s["draft_logits"] is not None:
                y = s["draft_logits"][i, t].double()
                lp = lp - (y[x] / T[i] - torch.logsumexp(y / T[i], 0))
            prob[i, t] = min(1.0, math.exp(float(lp)))
    return dict(tokens=None, accepted=None, prob=prob)


def _exact_linear4(c, seed):
    s = _prepare_linear4(c, seed)
    N, K, G = c["n"], c["k"], c["group"]
    y = torch.empty((c["rows"], N), dtype=torch.float64, device=DEV)
    x = s["x"].double()
    step = max(1, (1 << 27) // K)
    for a in range(0, N, step):
        w4 = s["w4"][a:a + step]
        w = torch.empty((w4.shape[0], K), dtype=torch.float64, device=DEV)
        w[:, 0::2], w[:, 1::2] = (w4 % 16).double(), (w4 // 16).double()
        z = s["zeros"][a:a + step].double() if s["zeros"] is not None else torch.full((w4.shape[0], K // G), 8.0, dtype=torch.float64, device=DEV)
        w = (w - z.repeat_interleave(G, 1)) * s["scales"][a:a + step].double().repeat_interleave(G, 1)
        y[:, a:a + step] = x @ w.t()
    return dict(y=y)


def exact(case, seed):
    return dict(append=_exact_append, sparse=_exact_sparse, verify=_exact_verify, linear4=_exact_linear4)[case["op"]](case, seed)
