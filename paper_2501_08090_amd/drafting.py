"""Draft and verify: speculative decoding of a model with a cheap copy of itself, over one paged cache.

The draft is the model with its matrices in 4 bits (`Linear4`) and attention over the cache pages that a cheap score selects
(`op_select_pages`, `op_sparse_attention`); it writes the keys and values of drafted tokens into the model's own pages
(`KVPool.append_rope`), where `decode_step_multi` overwrites them with the model's when it verifies.  `verify_drafts` accepts or
replaces.  The tokens that come out are distributed as the model's own samples (at temperature 0: they are its greedy tokens),
whatever the draft.

    python -m paper_2501_08090_amd.drafting --steps 16 --drafts 4

runs it on the two-layer toy decoder with random weights.
"""
import argparse
import math

import numpy as np
import torch

from . import binding as B
from . import inputs as I


def quantize4(w, group):
    """w [N, K] -> (w4 uint8 [N, K/2], scales bf16 [N, K/group]) with w ~ (q - 8) * scale: the group's largest value becomes 7 steps.
    K a multiple of group; a group of zeros has scale 0."""
    N, K = w.shape
    x = w.float().view(N, K // group, group)
    scales = (x.abs().amax(-1) / 7.0).to(torch.bfloat16)
    s = scales.float()[..., None]
    q = torch.where(s > 0, torch.round(x / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(x)).clamp(-8, 7).to(torch.int32) + 8
    q = q.view(N, K // 2, 2)
    return (q[..., 0] | q[..., 1] << 4).to(torch.uint8), scales


def _padded(w, rows, cols):
    out = torch.zeros((rows, cols), dtype=w.dtype, device=w.device)
    out[:w.shape[0], :w.shape[1]] = w
    return out


class Drafter:
    """The cheap copy.  w: the weights the model was loaded with (a dict as inputs.make_weights gives, on the GPU); matrices whose
    inputs are no multiple of `group` are padded with zeros."""

    def __init__(self, model, pool, w, group=128, top=64, n_first=1, n_last=1):
        cfg = model.cfg
        self.model, self.pool, self.top, self.n_first, self.n_last = model, pool, top, n_first, n_last
        self.index = B.KVIndex(pool)
        up = lambda n: -(-n // group) * group  # noqa: E731
        self.hidden, self.ffn, self.attn = up(cfg.hidden), up(cfg.ffn), up(cfg.n_q_heads * cfg.head_dim)
        lin = lambda m, rows, cols: B.Linear4(*quantize4(_padded(m, rows, cols), group))  # noqa: E731
        self.layers = []
        for l in range(cfg.n_layers):
            qkv = torch.cat((w["wq"][l], w["wk"][l], w["wv"][l]))
            self.layers.append(dict(
                qkv=lin(qkv, qkv.shape[0], self.hidden), o=lin(w["wo"][l], cfg.hidden, self.attn),
                gate_up=lin(torch.cat((_padded(w["w_gate"][l], self.ffn, self.hidden), _padded(w["w_up"][l], self.ffn, self.hidden))), 2 * self.ffn, self.hidden),
                down=lin(w["w_down"][l], cfg.hidden, self.ffn), attn_norm=w["attn_norm"][l], ffn_norm=w["ffn_norm"][l]))
        self.embed, self.final_norm = w["embed"], w["final_norm"]
        self.head = lin(w["lm_head"], cfg.vocab, self.hidden)

    def _norm(self, h, gain):
        x = B.op_rmsnorm(h, gain, self.model.cfg.rms_eps)
        return x if x.shape[1] == self.hidden else torch.nn.functional.pad(x, (0, self.hidden - x.shape[1]))

    def step(self, block_table, seq_lens, tokens):
        """One draft step: tokens [batch] at the positions seq_lens (tokens already cached) -> logits fp32 [batch, vocab].  Writes
        the tokens' keys and values, as the draft has them, into their pages."""
        cfg, batch = self.model.cfg, tokens.numel()
        qn, kn, d = cfg.n_q_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim, cfg.head_dim
        starts = torch.arange(batch + 1, dtype=torch.int32, device=tokens.device)
        cos, sin = B.rope_table(seq_lens, d, cfg.rope_base)
        ctx = seq_lens + 1
        h = self.embed[tokens.long()].float()
        for l, p in enumerate(self.layers):
            qkv = p["qkv"](self._norm(h, p["attn_norm"]))
            q, k, v = (t.unflatten(1, (-1, d)) for t in qkv.split((qn, kn, kn), 1))
            q = self.pool.append_rope(l, k, v, cos, sin, block_table, starts, seq_lens, q=q, index=self.index).view(batch, qn)
            pages, counts = B.op_select_pages(self.model, self.pool, self.index, l, q, block_table, ctx, self.top, n_first=self.n_first,
                                              n_last=self.n_last)
            a = B.op_sparse_attention(self.model, self.pool, l, q, block_table, ctx, pages, counts)
            if self.attn != qn:
                a = torch.nn.functional.pad(a, (0, self.attn - qn))
            p["o"](a, h, accumulate=True)
            g, u = p["gate_up"](self._norm(h, p["ffn_norm"])).split(self.ffn, 1)
            p["down"](torch.nn.functional.silu(g) * u, h, accumulate=True)
        return self.head(self._norm(h, self.final_norm))


def sample(logits, temperature, noise):
    """A token per row: argmax of softmax(logits / T) / noise over the tokens of a probability above 0, or of the logits where T is 0 (or
    no number above it).  The probabilities are those that verify_drafts takes a draft to be sampled from: NaN logits count as -inf,
    +inf as the largest finite value, 1 / T stays within fp32's range, and T = +inf leaves logits above -inf alike."""
    f = torch.finfo(torch.float32)
    z = torch.where(logits.isnan(), torch.full_like(logits, -math.inf), logits).clamp(max=f.max)
    top = z.amax(-1, keepdim=True)
    t = torch.where(temperature > 0, temperature, torch.ones_like(temperature))
    inv = (1.0 / t).clamp(f.tiny * f.eps, f.max)[:, None]
    w = torch.exp((z - torch.where(top.isinf(), torch.zeros_like(top), top)) * inv)
    race = torch.where(w > 0, w / w.sum(-1, keepdim=True) / noise, torch.full_like(w, -1.0))
    return torch.where((temperature > 0)[:, None], race, z).argmax(-1).to(torch.int32)


def draft_and_verify(drafter, block_table, seq_lens, tokens, drafts, temperature, generator):
    """One round: `drafts` tokens drafted behind tokens [batch], verified by one step of the model, accepted or replaced.
    -> new tokens int32 [batch, drafts+1] (accepted + 1 of them, then -1), accepted int32 [batch], and the next round's
    seq_lens and tokens (token 0 for a request whose logits left nothing to choose, where the new token is -1).  The pages of the positions seq_lens .. seq_lens+drafts must be in the block table."""
    model, pool = drafter.model, drafter.pool
    batch, vocab, dev = tokens.numel(), model.cfg.vocab, tokens.device
    fed, draft_logits = [tokens], []
    for t in range(drafts):
        logits = drafter.step(block_table, seq_lens + t, fed[-1])
        draft_logits.append(logits)
        fed.append(sample(logits, temperature, torch.empty((batch, vocab), device=dev).exponential_(generator=generator)))
    fed = torch.stack(fed, 1).contiguous()
    logits = B.decode_step_multi(model, pool, block_table, seq_lens, fed)
    uniforms = torch.rand((batch, drafts), generator=generator, device=dev)
    noise = torch.empty((batch, vocab), device=dev).exponential_(generator=generator)
    out, accepted, _ = B.verify_drafts(logits, fed[:, 1:].contiguous(), uniforms, noise,
                                       draft_logits=torch.stack(draft_logits, 1) if drafts else None, temperature=temperature)
    seq_next = seq_lens + accepted + 1
    drafter.index.update(block_table, seq_lens, seq_next, drafts + 1)  # the model's keys have taken the place of the draft's
    return out, accepted, seq_next, out.gather(1, accepted.long()[:, None]).view(-1).clamp(min=0)  # a step takes no token that is none


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=16, help="rounds of drafting and verifying")
    ap.add_argument("--drafts", type=int, default=4, help="drafted tokens a round")
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--context", type=int, default=600, help="cached tokens a request begins with")
    ap.add_argument("--top", type=int, default=16, help="pages a draft attends")
    ap.add_argument("--temperature", type=float, default=0.7)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    m = I.TINY
    lens = np.full(a.batch, a.context, np.int32)
    bt, blocks = I.make_block_table(lens + a.steps * (a.drafts + 1), seed=a.seed)
    model = B.Model(m, a.batch * (a.drafts + 1), bt.shape[1])
    w = I.make_weights(m, seed=a.seed, device="cuda")
    model.load_weights(w)
    pool = B.KVPool(model, num_blocks=blocks)
    block_table, seq_lens = torch.from_numpy(bt).cuda(), torch.from_numpy(lens).cuda()
    si, ps = I.prefill_index(lens)
    for l in range(m["n_layers"]):  # synthetic prompts
        k, v = I.make_kv_layer(m, len(si), l, seed=a.seed, device="cuda")
        pool.append(l, k, v, block_table, torch.from_numpy(si).cuda(), torch.from_numpy(ps).cuda())
    drafter = Drafter(model, pool, w, group=64, top=a.top)
    drafter.index.update(block_table, torch.zeros_like(seq_lens), seq_lens, a.context)
    g = torch.Generator(device="cuda")
    g.manual_seed(a.seed)
    tokens = torch.from_numpy(I.token_ids(a.batch, m["vocab"], a.seed)).cuda()
    temperature = torch.full((a.batch,), a.temperature, device="cuda")
    taken = 0
    for r in range(a.steps):
        out, accepted, seq_lens, tokens = draft_and_verify(drafter, block_table, seq_lens, tokens, a.drafts, temperature, g)
        taken += int(accepted.sum())
        print("round %2d: accepted %s of %d, new tokens %s" % (r, accepted.tolist(), a.drafts, [[t for t in row if t >= 0] for row in out.tolist()]))
    print("%.2f of %d drafted tokens accepted on average" % (taken / (a.steps * a.batch), a.drafts))


if __name__ == "__main__":
    main()
