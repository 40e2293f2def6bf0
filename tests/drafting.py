"""Definitions in 64 bits of the drafting operators (rotate-and-append, page index, page selection, attention over listed pages,
verification of drafts, 4-bit products), in plain numpy, and small caches to run them on."""
import math

import numpy as np
import torch

PAGE = 16
TOP32 = float(np.finfo(np.float32).max)
TOP16 = 3.3895313892515355e38  # the largest finite bf16


def power_of(amax):
    """exponent of the smallest power of two, at least 2^-126, with amax <= 127 * 2^e"""
    if amax == 0:
        return 0
    mant, e = math.frexp(float(amax))
    return max(-126, e - 7 + (1 if mant > 127 / 128 else 0))


def finite(x, top):
    return np.clip(np.nan_to_num(np.asarray(x, np.float64), nan=0.0, posinf=top, neginf=-top), -top, top)


def record(keys):
    """codes [2, d] and exponent of a page's keys [tokens, d]"""
    k = finite(keys, TOP16)
    hi, lo = k.max(0), k.min(0)
    e = power_of(max(abs(hi).max(), abs(lo).max()))
    return np.stack((np.ceil(np.ldexp(hi, -e)), np.floor(np.ldexp(lo, -e)))).astype(np.int64), e


def rotate(x, cos, sin):
    a, b = np.split(np.asarray(x, np.float64), 2, axis=-1)
    c, s = np.asarray(cos, np.float64)[:, None], np.asarray(sin, np.float64)[:, None]
    return np.concatenate((a * c - b * s, b * c + a * s), -1)


def select(q, codes, exps, ctx, top, n_first, n_last):
    """q [G, d], codes [pages, 2, d], exps [pages] of the row's pages -> ascending page list"""
    n = -(-max(ctx, 0) // PAGE)
    if n <= top:
        return list(range(n))
    x = finite(q, TOP32)
    q8 = np.rint(np.ldexp(x, -power_of(abs(x).max()))).astype(np.int64)
    dots = np.maximum(q8, 0) @ codes[:n, 0].T + np.minimum(q8, 0) @ codes[:n, 1].T
    score = np.clip(np.ldexp(dots.max(0).astype(np.float64), exps[:n]), -TOP32, TOP32)
    score[:n_first] = np.inf
    score[n - n_last:] = np.inf
    return sorted(np.argsort(-score, kind="stable")[:top].tolist())


def attend(q, k, v):
    """q [G, d] over k, v [tokens, d]; and how far the logits of a 32-bit computation can be off"""
    if len(k) == 0:
        return np.zeros_like(q), 0.0
    d = q.shape[1]
    x = q @ k.T / math.sqrt(d)
    w = np.exp(x - x.max(1, keepdims=True))
    slack = (d + 8) * 2.0 ** -24 * float((abs(q) @ abs(k).T).max()) / math.sqrt(d)
    return (w / w.sum(1, keepdims=True)) @ v, slack


def shares(z, t):
    z = np.where(np.isnan(z), -np.inf, np.minimum(np.asarray(z, np.float64), TOP32))
    m = z.max()
    if m == -np.inf:
        return np.zeros_like(z)
    w = np.exp((z - m) / t)
    return w / w.sum()


def verify(logits, tokens, uniforms, noise, draft_logits, n, temperature):
    """one request -> (tokens, accepted, prob, whether a decision is too near to call in 32 bits)"""
    drafts, V = len(tokens), logits.shape[1]
    prob, near = np.zeros(drafts), False
    clean = np.where(np.isnan(logits), -np.inf, np.minimum(logits.astype(np.float64), TOP32))
    best = [int(np.argmax(r)) if r.max() > -np.inf else -1 for r in clean]
    greedy = not temperature > 0
    for t in range(n):
        x = int(tokens[t])
        if not 0 <= x < V:
            continue
        if greedy:
            prob[t] = float(x == best[t])
            continue
        px = shares(logits[t], temperature)[x]
        if draft_logits is None:
            prob[t] = px
        else:
            qx = shares(draft_logits[t], temperature)[x]
            prob[t] = min(1.0, px / qx) if qx > 0 else float(px > 0)
    took = 0
    while took < n and float(uniforms[took]) < prob[took]:
        took += 1
    near |= any(prob[t] < 1 and abs(float(uniforms[t]) - prob[t]) < 1e-5 * max(prob[t], 1e-30) for t in range(min(n, took + 1)))
    if greedy:
        new = best[took]
    else:
        p = shares(logits[took], temperature)
        r = p
        if took < n:
            if draft_logits is not None:
                r = np.maximum(p - shares(draft_logits[took], temperature), 0)
            else:
                r = p.copy()
                if 0 <= tokens[took] < V:
                    r[tokens[took]] = 0
            if not (r > 0).any():
                r = p
            elif draft_logits is not None and r.max() < 1e-5:
                near = True  # what is left is rounding
        if not (r > 0).any():
            new = -1
        else:
            with np.errstate(divide="ignore"):
                race = np.where(r > 0, r / noise.astype(np.float64), -1.0)
            new = int(np.argmax(race))
            two = np.partition(race, -2)[-2] if V > 1 else -1.0
            near |= bool(two > race[new] * (1 - 1e-4))
    out = [int(x) for x in tokens[:took]] + [new] + [-1] * (drafts - took)
    return out, took, prob, near


def weights4(w4, scales, zeros, group):
    """[N, K] in 64 bits from packed nibbles, bf16 scales and zero points (torch tensors on the CPU)"""
    w4 = w4.numpy().astype(np.int64)
    q = np.stack((w4 & 15, w4 >> 4), -1).reshape(w4.shape[0], -1)
    z = np.full(scales.shape, 8) if zeros is None else zeros.numpy().astype(np.int64)
    s = scales.double().numpy()
    return (q - np.repeat(z, group, 1)) * np.repeat(s, group, 1), np.repeat(s, group, 1)


# ---- on the GPU (only the gpu tests call these) --------------------------------------------------------------------

class Cache:
    """A model handle, pool and page index of one or more layers, every slot NaN to begin with"""

    def __init__(self, n_q, n_kv, d, blocks, max_batch=64, max_blocks=64, layers=1, index=True):
        from paper_2501_08090_amd import binding as B
        m = dict(n_layers=layers, hidden=16, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=d, ffn=16, vocab=16, rope_base=10000.0, rms_eps=1e-5)
        self.model = B.Model(m, max_batch, max_blocks)
        mem = torch.empty(blocks * self.model.kv_block_bytes(), dtype=torch.uint8, device="cuda")
        mem.view(torch.int16).fill_(0x7FC0)
        self.pool = B.KVPool(self.model, memory=mem)
        assert self.pool.num_blocks == blocks
        self.index = None
        if index:
            from paper_2501_08090_amd.binding import load
            n = int(load().chiron_kv_index_bytes(self.pool._h))
            self.index = B.KVIndex(self.pool, memory=torch.full((n,), 0x55, dtype=torch.uint8, device="cuda"))
        self.n_q, self.n_kv, self.d, self.blocks, self.G = n_q, n_kv, d, blocks, n_q // n_kv

    def keys(self, layer=0):
        k, _ = self.pool.layer_views(layer)
        return k.reshape(self.blocks, PAGE, self.n_kv, self.d).double().cpu().numpy()

    def values(self, layer=0):
        _, v = self.pool.layer_views(layer)
        return v.reshape(self.blocks, PAGE, self.n_kv, self.d).double().cpu().numpy()

    def bits(self, layer=0):
        k, v = self.pool.layer_views(layer)
        f = lambda t: t.reshape(self.blocks, PAGE, self.n_kv, self.d).contiguous().view(torch.int16).cpu().numpy()  # noqa: E731
        return f(k), f(v)


def tables(lens, seed, extra=3):
    """distinct pages in random order, -1 elsewhere"""
    need = [-(-n // PAGE) for n in lens]
    rng = np.random.default_rng(seed)
    ids = rng.permutation(sum(need) + extra)
    bt = np.full((len(lens), max(max(need), 1)), -1, np.int32)
    o = 0
    for i, n in enumerate(need):
        bt[i, :n] = ids[o:o + n]
        o += n
    return bt, sum(need) + extra


def widen(bt, cols):
    out = np.full((bt.shape[0], cols), -1, np.int32)
    out[:, :bt.shape[1]] = bt
    return out


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()
