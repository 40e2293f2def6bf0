"""The operators of a long-context instance: what it calls for each new token, or each prompt, besides the projections, when its cache is
held in 8 bits or its layers see a window.

  tick     between two iterations: the pages of ended requests and of rejected drafts go back to the free list, the requests that go on and
           those that come in get the pages that their new tokens need, and the maps from rows to requests, positions and slots are laid out
  append8  keys and values of new tokens rotated, rounded to 8 bits with one power of two for each page and KV head, and written to
           their pages (what the page held before keeps its value, rounded again where the power of two has grown); queries rotated
  attend   one layer's attention of the new rows of each request, single tokens or whole prompts, over its cache: pages of 8-bit
           values (int8 or e4m3) or of bf16; causal, within a window and over a few first tokens that stay visible

`run` computes them in plain torch in 32 bits (`own` false) or by the framework's entry points (`own` true); `exact` in 64 bits.  What the
8-bit cache holds follows from the rotated keys by exact arithmetic; a rotation is two products and a sum, each rounded to 32 bits.
"""
import math
import random

import torch

own = False

PAGE = 16
LIMIT = 2.0 ** 100  # values in the 8-bit cache count as this where they are larger; steps are not finer than 1 / LIMIT
DEV = "cuda"


def _heads(q, kv, d):
    return dict(n_q_heads=q, n_kv_heads=kv, head_dim=d)


def listed():
    eight, small = _heads(32, 8, 128), _heads(16, 2, 64)
    return [
        # the benchmark's batch between two decode steps: two requests have ended and two prompts come in their place
        dict(name="tick_b64", op="tick", batch=64, width=512, median=800, prompts=2, drafts=0, scarce=False),
        # a large queue on an instance that drafts: rejected drafts give pages back, the free list does not hold what all of them ask for
        dict(name="tick_b1501_scarce", op="tick", batch=1501, width=1024, median=1000, prompts=60, drafts=5, scarce=True),
        # one decode step of the benchmark's batch: 64 requests bring one token each, fp32 rows of a fused projection
        dict(name="append8_b64", op="append8", batch=64, rows=64, median=800, dtype="f32", fmt="int8", **eight),
        # the prompts of 37 requests of very different lengths enter a layer, some behind a shared prefix
        dict(name="append8_ragged_5003", op="append8", batch=37, rows=5003, median=300, dtype="bf16", fmt="e4m3", **eight),
        # chunked prefill of four long prompts
        dict(name="append8_16k", op="append8", batch=4, rows=16384, median=2000, dtype="f32", fmt="int8", **eight),
        # one interactive user, 8k tokens: latency
        dict(name="attend8_b1_8k", op="attend", batch=1, lo=8000, hi=8192, new_lo=1, new_hi=1, window=0, sinks=0, fmt="int8", dtype="f32", **eight),
        # the long-document batch
        dict(name="attend8_b32_long32k", op="attend", batch=32, lo=24576, hi=32768, new_lo=1, new_hi=1, window=0, sinks=0, fmt="e4m3", dtype="f32", **eight),
        # chunks of three long prompts behind what is cached of them
        dict(name="attend8_chunks_12k", op="attend", batch=3, lo=11000, hi=12500, new_lo=500, new_hi=1100, window=0, sinks=0, fmt="int8", dtype="bf16", **eight),
        # several tokens of each request at once, other head geometry, lengths from nothing on
        dict(name="attend8_b61x5_ragged", op="attend", batch=61, lo=0, hi=5000, new_lo=0, new_hi=5, window=0, sinks=0, fmt="e4m3", dtype="f32", **small),
        # the long-document batch on layers with a window, bf16 cache
        dict(name="window_b32_long32k", op="attend", batch=32, lo=24576, hi=32768, new_lo=1, new_hi=1, window=4096, sinks=4, fmt="bf16", dtype="f32", **eight),
        # one long prompt through such a layer
        dict(name="window_prompt_8k", op="attend", batch=1, lo=0, hi=0, new_lo=8192, new_hi=8192, window=1024, sinks=4, fmt="bf16", dtype="bf16", **eight),
        # short prompts of odd lengths and single tokens together, a window that ends inside pages
        dict(name="window_b29_mixed", op="attend", batch=29, lo=0, hi=3000, new_lo=1, new_hi=333, window=777, sinks=5, fmt="bf16", dtype="f32", **small),
    ]


def _log(rng, lo, hi):
    """a whole number, spread evenly over the logarithm of the range"""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("tick", "append8", "attend", "attend"))
    if op == "tick":
        batch = _log(rng, 1, 1501)
        return dict(op=op, batch=batch, width=_log(rng, 16, 1024), median=_log(rng, 16, 1000), prompts=rng.randint(0, max(1, batch // 20)),
                    drafts=rng.choice((0, 0, 3, 5)), scarce=rng.random() < 0.3)
    kv = rng.choice((1, 2, 4, 8))
    heads = _heads(kv * rng.choice((1, 2, 4, 8, 16) if kv < 8 else (1, 2, 4)), kv, rng.choice((64, 128)))
    if op == "append8":
        rows = _log(rng, 1, 16384)
        return dict(op=op, batch=rng.randint(1, min(rows, 64)), rows=rows, median=_log(rng, 16, 2000), dtype=rng.choice(("f32", "bf16")),
                    fmt=rng.choice(("int8", "e4m3")), **heads)
    fmt, dtype = rng.choice(("int8", "e4m3", "bf16")), rng.choice(("f32", "bf16"))
    hi = _log(rng, 16, 32768)
    most = 450000000 // (heads["n_kv_heads"] * heads["head_dim"] * (2 if fmt == "bf16" else 1))  # tokens: half of the long-document batch
    batch = _log(rng, 1, max(1, min(64, most // hi)))
    kind = rng.choice(("one", "one", "few", "prompt"))
    new_hi = 1 if kind == "one" else rng.choice((2, 3, 5)) if kind == "few" else _log(rng, 17, 4096)
    # scores of the plain form and products of a pass: no more than the listed prompts have
    while new_hi > 1 and batch * heads["n_q_heads"] * new_hi * (hi + new_hi) > min(1 << 31, (110 << 30) // heads["head_dim"]):
        new_hi = max(1, new_hi // 2)
    window = rng.choice((0, _log(rng, 1, 8192))) if fmt != "bf16" else _log(rng, 1, 8192)
    return dict(op=op, batch=batch, lo=rng.choice((0, hi // 2)), hi=hi, new_lo=rng.choice((0, 1)) if new_hi > 1 and batch > 1 else 1, new_hi=new_hi, window=window,
                sinks=rng.choice((0, 1, 4, 17)) if window else 0, fmt=fmt, dtype=dtype, **heads)


# ---- inputs, made from the seed alone --------------------------------------------------------------------------

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + salt) & 0x7FFFFFFFFFFF)
    return g


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pages(n):
    return -(-n // PAGE)


def _tables(lens, seed):
    """distinct pages in random order for each request, -1 where it has none, and the number of pages of the pool"""
    need = [_pages(max(1, n)) for n in lens]
    total = sum(need)
    blocks = total + total // 8 + 1
    ids = torch.randperm(blocks, generator=torch.Generator().manual_seed(seed + 17))[:total].tolist()
    bt, o = [], 0
    for n in need:
        bt.append(ids[o:o + n] + [-1] * (max(need) - n))
        o += n
    return _i32(bt), blocks


def _handles(c, blocks, width):
    """the framework's pool for one layer of these heads: the handles that a program keeps"""
    from paper_2501_08090_amd import binding as B
    m = dict(n_layers=1, hidden=16, ffn=16, vocab=16, rope_base=10000.0, rms_eps=1e-5, **{k: c[k] for k in ("n_q_heads", "n_kv_heads", "head_dim")})
    model = B.Model(m, 1, width)
    return B.KVPool(model, num_blocks=blocks) if c.get("fmt") == "bf16" else B.KVPool8(model, num_blocks=blocks, format=c["fmt"])


def _views(c, k, v):
    """a plain cache [pages, 16, heads, d] in the shapes of the 8-bit or the bf16 pool's views"""
    nb, _, nkv, d = k.shape
    if c["fmt"] == "bf16":
        return k.view(nb, PAGE, nkv, d // 8, 8), v.view(nb, 4, 4, nkv, d // 32, 2, 16)
    return k.view(nb, PAGE, nkv, d // 16, 16), v.view(nb, 4, 4, nkv, d // 64, 4, 16)


def _cache(c, blocks, seed):
    """K and V of every page (codes and powers of two where they are held in 8 bits): keys of a page resemble each other, and a few of their
    dimensions are larger than the others"""
    g = _gen(seed, 1)
    shape = (blocks, PAGE, c["n_kv_heads"], c["head_dim"])
    if c["fmt"] == "bf16":
        k = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
        k.mul_(0.8).add_(torch.randn((blocks, 1) + shape[2:], generator=g, device=DEV, dtype=torch.bfloat16), alpha=0.6)
        return dict(K=k, V=torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16))
    s = {}
    for name in ("K", "V"):
        x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
        if name == "K":
            x.mul_(0.8).add_(torch.randn((blocks, 1) + shape[2:], generator=g, device=DEV, dtype=torch.bfloat16), alpha=0.6)
            x[..., 3] *= 4.0
        e = -4 if c["fmt"] == "int8" else -6
        x.mul_(2.0 ** -e)
        s[name] = torch.round(x).clamp_(-127, 127).to(torch.int8) if c["fmt"] == "int8" else x.clamp_(-448, 448).to(torch.float8_e4m3fn)
        # pages differ in how large their values are
        e = torch.randint(e - 1, e + 2, (blocks, c["n_kv_heads"]), generator=g, device=DEV, dtype=torch.int32)
        s["e" + name] = e
    return s


def _own_cache(s, c, blocks, width):
    """the same cache in the framework's pool"""
    s["pool"] = _handles(c, blocks, width)
    views = s["pool"].layer_views(0)
    for a, b in zip(views, _views(c, s.pop("K"), s.pop("V"))):
        (a if c["fmt"] == "bf16" else a.view(torch.int8)).copy_(b if c["fmt"] == "bf16" else b.view(torch.int8))
    if c["fmt"] != "bf16":
        views[2][..., 0].copy_(s.pop("eK"))
        views[2][..., 1].copy_(s.pop("eV"))


def _append_lens(c):
    r = random.Random(17)  # the lengths are the case's own, in an order that goes by the seed
    B_, rows = c["batch"], c["rows"]
    share = [math.exp(r.gauss(0, 1.5)) if rows > B_ else 1.0 for _ in range(B_)]
    new = [1 + int((rows - B_) * s / sum(share)) for s in share]
    new[0] += rows - sum(new)
    old = [min(4096, int(c["median"] * math.exp(r.gauss(0, 0.8)))) if r.random() < 0.8 else 0 for _ in range(B_)]
    return old, new


def _attend_lens(c):
    r = random.Random(19)
    old = [r.randint(c["lo"], c["hi"]) for _ in range(c["batch"])]
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["batch"])]
    if c["batch"] > 8 and c["lo"] == 0:
        old[1], old[2] = 0, 1
    if sum(new) == 0:
        new[0] = 1
    return old, new


def _rows(old, new, seed):
    """the requests in an order that goes by the seed, their block table and row starts"""
    order = random.Random(seed).sample(range(len(old)), len(old))
    old, new = [old[i] for i in order], [new[i] for i in order]
    bt, blocks = _tables([a + b for a, b in zip(old, new)], seed)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    return dict(block_table=bt, row_starts=_i32(starts), seq_lens=_i32(old), n_rows=starts[-1], max_new=max(new)), blocks, old, new


def _prepare_append(c, seed):
    rows, d, nq, nkv = c["rows"], c["head_dim"], c["n_q_heads"], c["n_kv_heads"]
    s, blocks, old, new = _rows(*_append_lens(c), seed)
    g = _gen(seed, 2)
    qkv = torch.randn((rows, (nq + 2 * nkv) * d), generator=g, device=DEV, dtype=torch.float32)
    if c["dtype"] == "bf16":
        qkv = qkv.to(torch.bfloat16)
    s.update(case=c, q=qkv[:, :nq * d].unflatten(1, (nq, d)), k=qkv[:, nq * d:(nq + nkv) * d].unflatten(1, (nkv, d)),
             v=qkv[:, (nq + nkv) * d:].unflatten(1, (nkv, d)))
    pos = torch.cat([torch.arange(o, o + n) for o, n in zip(old, new)]).to(DEV)
    angle = pos.double()[:, None] * 500000.0 ** (-2.0 * torch.arange(d // 2, device=DEV).double() / d)
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    # what a pass reads back: the new tokens, and the old ones of the pages that the first of them come to
    look = [(i, p) for i, (o, n) in enumerate(zip(old, new)) for p in range(o // PAGE * PAGE if n else o, o + n)]
    s["look_seq"], s["look_pos"] = _i32([i for i, _ in look]), _i32([p for _, p in look])
    s.update(_cache(c, blocks, seed))
    return s, blocks


def _prepare_attend(c, seed):
    s, blocks, old, new = _rows(*_attend_lens(c), seed)
    g = _gen(seed, 2)
    q = torch.randn((s["n_rows"], c["n_q_heads"], c["head_dim"]), generator=g, device=DEV, dtype=torch.float32) * 1.5
    s.update(case=c, q=q.to(torch.bfloat16) if c["dtype"] == "bf16" else q)
    s.update(_cache(c, blocks, seed))
    return s, blocks


def _tick_lens(c):
    """tokens kept and new ones of each request, and how many pages the table holds for it now"""
    r = random.Random(23)
    B_, top = c["batch"], c["width"] * PAGE
    keep, new, has = [], [], []
    coming = set(r.sample(range(B_), min(B_, c["prompts"])))
    for i in range(B_):
        n = max(1, min(top - 8, int(c["median"] * math.exp(r.gauss(0, 1.0)))))
        if i in coming:  # an ended request's row, taken by a prompt
            m = max(1, min(top, int((3 if c["scarce"] else 1) * c["median"] * math.exp(r.gauss(0, 1.0)))))
            keep.append(0), new.append(m), has.append(_pages(n))
        else:
            t = 1 + (r.randint(0, c["drafts"]) if c["drafts"] else 0)
            keep.append(n), new.append(t), has.append(_pages(min(top, n + c["drafts"])))
    return keep, new, has


def _prepare_tick(c, seed):
    keep, new, has = _tick_lens(c)
    order = random.Random(seed).sample(range(len(keep)), len(keep))
    keep, new, has = [keep[i] for i in order], [new[i] for i in order], [has[i] for i in order]
    ask = sum(_pages(a + b) - _pages(a) for a, b in zip(keep, new))
    back = sum(max(0, h - _pages(a)) for a, h in zip(keep, has))
    spare = max(0, ask // 2 - back) if c["scarce"] else max(0, ask - back) + 100
    blocks = sum(has) + spare
    ids = torch.randperm(blocks, generator=torch.Generator().manual_seed(seed + 29)).to(torch.int32)
    bt, o = torch.full((c["batch"], c["width"]), -1, dtype=torch.int32), 0
    for i, h in enumerate(has):
        bt[i, :h] = ids[o:o + h]
        o += h
    free = torch.zeros(blocks, dtype=torch.int32)
    free[:spare] = ids[o:]
    s = dict(case=c, block_table=bt.to(DEV), keep=_i32(keep), new=_i32(new), max_rows=sum(new) + 8)
    if own:
        from paper_2501_08090_amd import binding as B
        s["pages"] = B.PageList(free.to(DEV), _i32([spare]))
    else:
        s["free"], s["count"] = free.to(DEV), _i32([spare])
    return s


def prepare(case, seed):
    op = case["op"]
    if op == "tick":
        return _prepare_tick(case, seed)
    s, blocks = (_prepare_append if op == "append8" else _prepare_attend)(case, seed)
    if own:
        _own_cache(s, case, blocks, s["block_table"].shape[1])
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------

def _two(e):
    """2^e as an exact fp32 value, -126 <= e <= 127"""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _power(amax, fmt):
    """the exponent e of the smallest power of two, at least 1 / LIMIT, with amax <= 127 * 2^e, or 448 * 2^e for e4m3"""
    mant, ex = torch.frexp(amax)
    e = ex - 7 + (mant > 127.0 / 128.0) if fmt == "int8" else ex - 9 + (mant > 448.0 / 512.0)
    return torch.where(amax > 0, e, torch.full_like(e, -100)).clamp(min=-100)


def _bounded(x):
    return torch.where(torch.isnan(x), torch.zeros_like(x), x).clamp(-LIMIT, LIMIT)


def _rounded(x, fmt):
    """x, at most the format's largest value, to the nearest value of the format, ties to even"""
    if fmt == "int8":
        return torch.round(x).to(torch.int8)
    step = torch.frexp(x)[1].clamp(min=-5) - 4
    return (torch.round(x * _two(-step)) * _two(step)).to(torch.float8_e4m3fn)


def _rotate(x, cos, sin):
    """pairs (j, j + d/2) of x [rows, heads, d] turned by their row's angles"""
    x = x.float()
    a, b = x.chunk(2, -1)
    c, s = cos[:, None, :], sin[:, None, :]
    return torch.cat((a * c - b * s, b * c + a * s), -1)


def _store8(codes, exps, x, page, slot, part, fmt):
    """x [rows, heads, d] into (page, slot) of codes; part: pages that hold old tokens"""
    x = _bounded(x)
    amax = x.abs().amax(-1)
    top = torch.zeros_like(exps, dtype=torch.float32)
    top.scatter_reduce_(0, page[:, None].expand_as(amax), amax, "amax")
    before = torch.full_like(exps, -100)
    before[part] = exps[part]
    e = torch.maximum(_power(top, fmt), before)
    moved = codes[part].float() * _two((exps[part] - e[part]).clamp(min=-126))[:, None, :, None]
    codes[part] = _rounded(moved, fmt)
    codes[page, slot] = _rounded(x * _two(-e[page])[..., None], fmt)
    exps[page] = e[page]


def _values(codes, exps, page, slot):
    """what slots hold: exact in bf16"""
    return (codes[page, slot].float() * _two(exps[page])[..., None]).to(torch.bfloat16)


def _append_plain(s):
    fmt = s["case"]["fmt"]
    rows = s["q"].shape[0]
    row = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(s["row_starts"].long(), row, right=True) - 1
    pos = s["seq_lens"].long()[seq] + row - s["row_starts"].long()[seq]
    page, slot = s["block_table"].long()[seq, pos // PAGE], pos % PAGE
    old = s["seq_lens"].long()
    # the page that a request's first new token shares with old ones
    first = s["block_table"].long()[torch.arange(old.numel(), device=DEV), (old // PAGE).clamp(max=s["block_table"].shape[1] - 1)]
    part = first[(old % PAGE > 0) & (s["row_starts"][1:] > s["row_starts"][:-1])]
    _store8(s["K"], s["eK"], _rotate(s["k"], s["cos"], s["sin"]), page, slot, part, fmt)
    _store8(s["V"], s["eV"], s["v"].float(), page, slot, part, fmt)
    at = s["look_pos"].long()
    page, slot = s["block_table"].long()[s["look_seq"].long(), at // PAGE], at % PAGE
    k, v = (_values(s[n], s["e" + n], page, slot) for n in ("K", "V"))
    return dict(q=_rotate(s["q"], s["cos"], s["sin"]), k=k, v=v)


def _spans(s):
    """positions [batch, span] that some row of a request may see, and how many there are: the first tokens, then the union of the rows' windows"""
    c = s["case"]
    old, starts = s["seq_lens"].long(), s["row_starts"].long()
    n = starts[1:] - starts[:-1]
    end = old + n
    if c["window"]:
        begin = (old - c["window"] + 1).clamp(min=0)
        first = torch.minimum(begin, torch.full_like(begin, c["sinks"]))
        width = min(c["hi"] + s["max_new"], c["sinks"] + c["window"] + s["max_new"])
    else:
        begin = first = torch.zeros_like(old)
        width = c["hi"] + s["max_new"]
    j = torch.arange(width, device=DEV)[None, :]
    pos = torch.where(j < first[:, None], j, begin[:, None] + j - first[:, None])
    return pos, pos < end[:, None]


def _attend_plain(s):
    c = s["case"]
    d, nkv, nq = c["head_dim"], c["n_kv_heads"], c["n_q_heads"]
    G, N, rows = nq // nkv, s["max_new"], s["q"].shape[0]
    starts, old = s["row_starts"].long(), s["seq_lens"].long()
    B_ = old.numel()
    t = torch.arange(N, device=DEV)
    q = s["q"][(starts[:-1, None] + t).clamp(max=rows - 1)].float().view(B_, N, nkv, G, d).permute(0, 2, 3, 1, 4).reshape(B_, nkv, G * N, d)
    pos, there = _spans(s)
    page = s["block_table"].long().gather(1, (pos // PAGE).clamp(max=s["block_table"].shape[1] - 1)).clamp(min=0)
    slot = pos % PAGE

    def taken(name):
        x = s[name][page, slot].float()
        if "e" + name in s:
            x = x * _two(s["e" + name])[page][..., None]
        return x.permute(0, 2, 1, 3)

    k = taken("K").contiguous()
    x = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(d)
    del k
    at = (old[:, None] + t)[:, :, None]  # the rows' own positions
    live = there[:, None, :] & (pos[:, None, :] <= at)
    if c["window"]:
        live = live & ((pos[:, None, :] > at - c["window"]) | (pos[:, None, :] < c["sinks"]))
    x = x.view(B_, nkv, G, N, -1).masked_fill_(~live[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    w = x.sub_(torch.where(torch.isinf(m), torch.zeros_like(m), m)).exp_()
    z = w.sum(-1, keepdim=True)
    v = torch.where(there[:, None, :, None], taken("V"), torch.zeros((), device=DEV))
    out = torch.matmul(w.view(B_, nkv, G * N, -1), v).view(B_, nkv, G, N, d) / torch.where(z > 0, z, torch.ones_like(z))
    row = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(starts, row, right=True) - 1
    return out.permute(0, 3, 1, 2, 4)[seq, row - starts[seq]].reshape(rows, nq, d).to(s["q"].dtype)


def _tick_plain(s):
    bt, free, count = s["block_table"], s["free"], s["count"]
    keep, new = s["keep"].long(), s["new"].long()
    B_, width = bt.shape
    n = free.numel()
    col = torch.arange(width, device=DEV)[None, :]
    # what lies behind the tokens kept goes to the end of the free list, requests and columns in order
    back = (bt >= 0) & (col >= (keep[:, None] + PAGE - 1) // PAGE)
    rank = back.view(-1).long().cumsum(0)
    to = torch.where(back.view(-1), count.long() + rank - 1, torch.full_like(rank, n))
    grown = torch.nn.functional.pad(free, (0, 1))
    grown[to] = bt.view(-1)
    free.copy_(grown[:n])
    count += rank[-1:].to(torch.int32)
    bt.masked_fill_(back, -1)
    # what the new tokens need: a page for each of their columns that has none
    ask = (bt < 0) & (col >= keep[:, None] // PAGE) & (col < (keep + new + PAGE - 1)[:, None] // PAGE)
    fits = keep + new <= width * PAGE
    ask &= fits[:, None]
    need = ask.sum(1)
    tokens = torch.where(fits, new, torch.zeros_like(new))
    admitted = fits & (tokens.cumsum(0) <= s["max_rows"]) & ((need == 0) | (need.cumsum(0) <= count.long()))
    granted = torch.where(admitted, new, torch.zeros_like(new))
    ask &= admitted[:, None]
    total = ask.sum()
    rank = ask.view(-1).long().cumsum(0)
    given = free[(count.long() - total + rank - 1).clamp(0, n - 1)].view(B_, width)
    bt.copy_(torch.where(ask, given, bt))
    count -= total.to(torch.int32)
    starts = torch.nn.functional.pad(granted.cumsum(0), (1, 0))
    row = torch.arange(s["max_rows"], device=DEV)
    seq = torch.searchsorted(starts, row, right=True) - 1
    live = row < starts[-1]
    seq = torch.where(live, seq, torch.zeros_like(seq))
    pos = torch.where(live, keep[seq] + row - starts[seq], torch.zeros_like(row))
    slots = bt[seq, pos // PAGE].long() * PAGE + pos % PAGE
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return dict(block_table=bt, free=free, count=count, row_starts=i32(starts), row_seq=i32(torch.where(live, seq, torch.full_like(seq, -1))),
                pos=i32(pos), slots=torch.where(live, slots, torch.full_like(slots, -1)), granted=i32(granted))


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "append8":
            return _append_plain(s)
        return _tick_plain(s) if op == "tick" else dict(out=_attend_plain(s))
    from paper_2501_08090_amd import binding as B
    if op == "tick":
        pages, bt = s["pages"], s["block_table"]
        pages.release(bt, s["keep"])
        m = pages.grant(bt, s["keep"], s["new"], s["max_rows"])
        return dict(block_table=bt, free=pages.pages, count=pages.count, row_starts=m.row_starts, row_seq=m.row_seq, pos=m.pos, slots=m.slots,
                    granted=m.granted)
    if op == "append8":
        pool = s["pool"]
        q = pool.append_rope(0, s["k"], s["v"], s["cos"], s["sin"], s["block_table"], s["row_starts"], s["seq_lens"], q=s["q"])
        k, v = pool.gather(0, s["block_table"], s["look_seq"], s["look_pos"])
        return dict(q=q, k=k, v=v)
    return dict(out=B.op_row_attention(s["pool"], 0, s["q"], s["block_table"], s["row_starts"], s["seq_lens"], window=s["case"]["window"],
                                       n_sinks=s["case"]["sinks"], max_new=s["max_new"]))


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def _seen(c, old, new):
    """positions that a request's rows read together, and the sum of what each sees"""
    w, k = c["window"], c["sinks"]
    if not w:
        return (old + new if new else 0), sum(old + t + 1 for t in range(new))
    each = sum(min(p + 1, w) + min(k, max(0, p + 1 - w)) for p in range(old, old + new))
    begin = max(0, old - w + 1)
    return (old + new - begin + min(k, begin) if new else 0), each


def work(c):
    op = c["op"]
    if op == "tick":
        keep, new, has = _tick_lens(c)
        moved = sum(max(0, h - _pages(a)) + _pages(a + b) - _pages(a) for a, b, h in zip(keep, new, has))
        # the table and the lengths in, the pages that move in and out, starts, rows, positions and slots out
        return dict(bytes=4 * c["batch"] * c["width"] + 12 * c["batch"] + 8 * moved + 16 * sum(new), flops=c["batch"] * c["width"])
    if op == "append8":
        q, kv = c["n_q_heads"] * c["head_dim"], 2 * c["n_kv_heads"] * c["head_dim"]
        size = 4 if c["dtype"] == "f32" else 2
        # rows in; rotated queries, keys and values out, and read back as bf16; the rotary table; a power of two for each page, head and side
        per_row = (q + kv) * size + 4 * q + kv + 3 * kv + 4 * c["head_dim"]
        return dict(bytes=c["rows"] * per_row + _pages(c["rows"]) * c["n_kv_heads"] * 2, flops=3 * c["rows"] * (q + kv // 2))
    seen = [_seen(c, a, b) for a, b in zip(*_attend_lens(c))]
    d, nq, nkv = c["head_dim"], c["n_q_heads"], c["n_kv_heads"]
    size, rows = 2 if c["fmt"] == "bf16" else 1, sum(_attend_lens(c)[1])
    return dict(bytes=sum(a for a, _ in seen) * nkv * d * 2 * size + rows * nq * d * (8 if c["dtype"] == "f32" else 4),
                flops=4 * d * nq * sum(b for _, b in seen))


# ---- the same in 64 bits, written apart ------------------------------------------------------------------------

def _exact_append(c, seed):
    s, blocks = _prepare_append(c, seed)
    fmt, half = c["fmt"], c["head_dim"] // 2
    starts, old, bt = s["row_starts"].tolist(), s["seq_lens"].tolist(), s["block_table"].tolist()
    cos, sin = s["cos"].double()[:, None], s["sin"].double()[:, None]

    def turned(x):
        x = x.double()
        y = torch.empty_like(x)
        y[..., :half] = x[..., :half] * cos - x[..., half:] * sin
        y[..., half:] = x[..., half:] * cos + x[..., :half] * sin
        return y

    def two(e):
        return ((e.long() + 1023) << 52).view(torch.float64)

    def nearest(x):
        if fmt == "int8":
            return torch.round(x)
        unit = two(torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 4)
        return torch.round(x / unit) * unit

    def stored(name, x):
        """values of the slots that a pass reads back, page by page"""
        top, found = 127.0 if fmt == "int8" else 448.0, []
        for i in range(c["batch"]):
            end = old[i] + starts[i + 1] - starts[i]
            for pg in range(old[i] // PAGE, (end - 1) // PAGE + 1):
                a, b, page = max(old[i], pg * PAGE), min(end, pg * PAGE + PAGE), bt[i][pg]
                new = x[starts[i] + a - old[i]:starts[i] + b - old[i]]
                was = s["e" + name][page].long()
                held = s[name][page, :a % PAGE].double() * two(was)[None, :, None]
                e = torch.ceil(torch.log2(new.abs().amax((0, 2)).clamp(min=1e-30) / top)).clamp(min=-100).long()
                unit = two(torch.maximum(e, was) if a % PAGE else e)[None, :, None]
                found.append(nearest(torch.cat((held, new)) / unit) * unit)
        return torch.cat(found)

    return dict(q=turned(s["q"]), k=stored("K", turned(s["k"])), v=stored("V", s["v"].double()))


def _exact_attend(c, seed):
    s, blocks = _prepare_attend(c, seed)
    d, nkv = c["head_dim"], c["n_kv_heads"]
    G = c["n_q_heads"] // nkv
    starts, old = s["row_starts"].tolist(), s["seq_lens"].tolist()
    out = torch.zeros((s["n_rows"], nkv, G, d), dtype=torch.float64, device=DEV)
    for i in range(c["batch"]):
        n = starts[i + 1] - starts[i]
        if n == 0:
            continue
        p = torch.arange(old[i] + n, device=DEV)
        page = s["block_table"][i].long()[p // PAGE]

        def cached(name):
            x = s[name][page, p % PAGE].double()
            return x * torch.ldexp(torch.ones_like(x[..., :1]), s["e" + name][page][..., None]) if "e" + name in s else x

        k, v = cached("K"), cached("V")
        at = torch.arange(old[i], old[i] + n, device=DEV)[:, None]
        hidden = p[None, :] > at
        if c["window"]:
            hidden = hidden | ((p[None, :] <= at - c["window"]) & (p[None, :] >= c["sinks"]))
        for h in range(nkv):
            for a in range(G):
                x = s["q"][starts[i]:starts[i + 1], h * G + a].double() @ k[:, h].t() / math.sqrt(d)
                out[starts[i]:starts[i + 1], h, a] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ v[:, h]
    return dict(out=out.view(s["n_rows"], c["n_q_heads"], d))


def exact(case, seed):
    if case["op"] == "tick":
        return None  # whole numbers
    return (_exact_append if case["op"] == "append8" else _exact_attend)(case, seed)
