"""Definitions in 64 bits of the long-context operators (page lists, the cache in 8 bits, attention of new rows within windows), in plain
numpy, and small caches to run them on."""
import math

import numpy as np
import torch

from drafting import PAGE, dev, rotate, tables, widen  # noqa: F401

LIMIT, MIN_EXP = 2.0 ** 100, -100
TOP = {"int8": 127.0, "e4m3": 448.0}


# ---- page lists ------------------------------------------------------------------------------------------------------

def release(bt, pages, first, end=None):
    """bt [requests, width] and the list of free pages, after: in place and returned"""
    pages = list(pages)
    for i in range(bt.shape[0]):
        c0 = -(-max(int(first[i]), 0) // PAGE)
        c1 = bt.shape[1] if end is None else min(max(int(end[i]), 0) // PAGE, bt.shape[1])
        for c in range(c0, c1):
            if bt[i, c] >= 0:
                pages.append(int(bt[i, c]))
                bt[i, c] = -1
    return pages


def grant(bt, pages, old, new, max_rows):
    """-> the list, row_starts, row_seq, pos, slots, granted; bt in place"""
    width = bt.shape[1]
    asked = need_so_far = 0
    wants, granted = [], []
    for o, n in zip(map(int, old), map(int, new)):
        fits = o >= 0 and n >= 0 and o + n <= width * PAGE
        i = len(wants)
        cols = [c for c in range(o // PAGE, -(-(o + n) // PAGE)) if bt[i, c] < 0] if fits and n else []
        asked += n if fits else 0
        need_so_far += len(cols)
        ok = fits and asked <= max_rows and (not cols or need_so_far <= len(pages))
        wants.append(cols if ok else [])
        granted.append(n if ok else 0)
    total = sum(map(len, wants))
    taken, left = pages[len(pages) - total:], pages[:len(pages) - total]
    k = 0
    for i, cols in enumerate(wants):
        for c in cols:
            bt[i, c] = taken[k]
            k += 1
    starts = np.concatenate([[0], np.cumsum(granted)]).astype(np.int64)
    seq, pos, slots = np.full(max_rows, -1), np.zeros(max_rows, np.int64), np.full(max_rows, -1, np.int64)
    for i, n in enumerate(granted):
        for t in range(n):
            r, p = int(starts[i]) + t, int(old[i]) + t
            seq[r], pos[r] = i, p
            if bt[i, p // PAGE] >= 0:
                slots[r] = int(bt[i, p // PAGE]) * PAGE + p % PAGE
    return left, starts, seq, pos, slots, np.array(granted)


# ---- 8 bits -----------------------------------------------------------------------------------------------------------

def bounded(x):
    x = np.asarray(x, np.float64)
    return np.clip(np.where(np.isnan(x), 0.0, x), -LIMIT, LIMIT)


def power(amax, fmt):
    if amax == 0:
        return MIN_EXP
    e = math.frexp(float(amax))[1] - 12
    while amax > TOP[fmt] * 2.0 ** e:
        e += 1
    return max(e, MIN_EXP)


def nearest(x, fmt):
    """values of the format nearest to x, ties to even"""
    if fmt == "int8":
        return np.rint(x)
    unit = np.ldexp(1.0, np.frexp(np.maximum(abs(x), 2.0 ** -6))[1] - 4)
    return np.rint(x / unit) * unit


def store(held, e_old, new, fmt):
    """values of a page's old tokens [n, d] and its exponent (ignored without old tokens), new values [m, d] -> values, exponent"""
    new = bounded(new)
    e = power(abs(new).max() if new.size else 0, fmt)
    if len(held):
        e = max(e, int(e_old))
    unit = 2.0 ** e
    return np.concatenate((nearest(held / unit, fmt) * unit, nearest(new / unit, fmt) * unit)), e


# ---- attention ----------------------------------------------------------------------------------------------------------

def visible(p, n_keys, window, sinks):
    u = np.arange(n_keys)
    return (u <= p) & ((u > p - window) | (u < sinks) if window else True)


def attend(q, k, v, see):
    """q [G, d] over k, v [tokens, d], of which `see` -> out, and how far the logits of a 32-bit computation can be off"""
    if not see.any():
        return np.zeros_like(q), 0.0
    k, v, d = k[see], v[see], q.shape[1]
    x = q @ k.T / math.sqrt(d)
    w = np.exp(x - x.max(1, keepdims=True))
    slack = (d + 8) * 2.0 ** -24 * float((abs(q) @ abs(k).T).max()) / math.sqrt(d)
    return (w / w.sum(1, keepdims=True)) @ v, slack


# ---- on the GPU (only the gpu tests call these) ---------------------------------------------------------------------------

class Cache:
    """A pool of one format, every slot NaN (bf16, e4m3) or of the largest code and exponent (int8) to begin with"""

    def __init__(self, n_kv, d, blocks, fmt, layers=1):
        from paper_2501_08090_amd import binding as B
        m = dict(n_layers=layers, hidden=16, n_q_heads=n_kv, n_kv_heads=n_kv, head_dim=d, ffn=16, vocab=16, rope_base=10000.0, rms_eps=1e-5)
        self.model = B.Model(m, 1, 8)
        self.fmt, self.n_kv, self.d, self.blocks = fmt, n_kv, d, blocks
        if fmt == "bf16":
            mem = torch.empty(blocks * self.model.kv_block_bytes(), dtype=torch.uint8, device="cuda")
            mem.view(torch.int16).fill_(0x7FC0)
            self.pool = B.KVPool(self.model, memory=mem)
        else:
            n = int(B.load().chiron_kv8_pool_bytes(self.model._h, blocks))
            self.pool = B.KVPool8(self.model, blocks, fmt, memory=torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda"))

    def values(self, layer=0):
        """K and V [blocks, 16, heads, d] in 64 bits"""
        shape = (self.blocks, PAGE, self.n_kv, self.d)
        if self.fmt == "bf16":
            return tuple(t.reshape(shape).double().cpu().numpy() for t in self.pool.layer_views(layer))
        k, v, e = self.pool.layer_views(layer)
        e = e.cpu().numpy().astype(np.int64)
        return tuple(np.ldexp(t.reshape(shape).float().double().cpu().numpy(), e[:, None, :, j, None]) for j, t in enumerate((k, v)))

    def fill(self, bt, lens, rng, layer=0, hot=True):
        """random tokens 0 .. lens[i]-1 of each request, other slots as they are"""
        k, v = (t for t in self.pool.layer_views(layer)[:2])
        shape = (self.blocks, PAGE, self.n_kv, self.d)
        for j, t in enumerate((k, v)):
            x = torch.from_numpy(rng.standard_normal(shape) * (1.0 + rng.random((self.blocks, 1, self.n_kv, 1)))).to(torch.bfloat16)
            if hot and j == 0:
                x[..., 1] *= 6.0
            live = torch.zeros(shape, dtype=torch.bool)
            for i, n in enumerate(lens):
                for c in range(-(-n // PAGE)):
                    if bt[i, c] >= 0:
                        live[bt[i, c], :min(PAGE, n - c * PAGE)] = True
            live = live.view(t.shape).cuda()
            if self.fmt == "bf16":
                t.copy_(torch.where(live, x.view(t.shape).cuda(), t))
                continue
            unit = 8.0 if self.fmt == "int8" else 32.0
            x = (x.float() * unit).clamp(-TOP[self.fmt], TOP[self.fmt])
            x = (torch.round(x).to(torch.int8) if self.fmt == "int8" else x.to(torch.float8_e4m3fn)).view(torch.int8)
            raw = t.view(torch.int8)
            raw.copy_(torch.where(live, x.view(t.shape).cuda(), raw))
            e = self.pool.layer_views(layer)[2]
            pages = live.reshape(shape)[:, 0, :, 0]
            pow2 = torch.from_numpy(rng.integers(-1, 2, (self.blocks, self.n_kv)) - int(math.log2(unit))).to(torch.int8).cuda()
            e[..., j].copy_(torch.where(pages, pow2, e[..., j]))
