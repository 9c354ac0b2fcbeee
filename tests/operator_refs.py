"""Plain references in 64 bits for the operators beside the step, and the error bounds that their types allow.

A rounding to bf16 is off by at most half a step, 2^-8 of the value, one to fp32 by 2^-24."""
import math

import numpy as np
import torch

F8 = torch.float64
BF16_HALF = 2.0 ** -8
PAGE = 16


def cuda(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


def context(**kw):
    from paper_2511_21699_b200 import Cacheback
    d = dict(batch=1, LL=1, FL=1, LC=1, FC=1, max_nodes=1, crt=0, max_depth=1, vocab=1, n_q_heads=1, n_kv_heads=1, head_dim=64)
    d.update(kw)
    return Cacheback(**d)


def rope_table(positions, rot, device="cuda"):
    ang = torch.arange(positions, device=device, dtype=F8)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device=device, dtype=F8) / rot)
    return torch.cat((ang.cos(), ang.sin()), 1).float()


def normed_and_turned(x, w, eps, table, pos, interleaved):
    """(value, bound on the error of a result rounded once to bf16) of [rows, heads, D] bf16 x."""
    y = x.to(F8)
    D = y.shape[-1]
    if w is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * w.to(F8)
    z, mag = y, y.abs()
    if table is not None:
        R = table.shape[1]
        c, s = table[pos, None, :R // 2].to(F8), table[pos, None, R // 2:].to(F8)
        ia = torch.arange(0, R, 2, device=x.device) if interleaved else torch.arange(R // 2, device=x.device)
        ib = ia + 1 if interleaved else ia + R // 2
        a, b = y[..., ia], y[..., ib]
        z, mag = y.clone(), y.abs()
        z[..., ia], z[..., ib] = a * c - b * s, b * c + a * s
        mag[..., ia], mag[..., ib] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    # in fp32: the sum of squares in D / 16 lanes of 16 (at most 16 + 3 roundings), its root, two products and the rotation's three: under 32 roundings of 2^-24
    return z, BF16_HALF * z.abs() + 32 * 2.0 ** -24 * (1 + BF16_HALF) * mag


class Paged:
    """Sequences in a paged cache: new and cached tokens of each, shuffled pages, a few spare ones."""

    def __init__(self, new, ctx, hkv, d, seed=0, spare_pages=1, width=None):
        self.new, self.ctx = np.asarray(new, np.int64), np.asarray(ctx, np.int64)
        need = -(-(self.new + self.ctx) // PAGE)
        rng = np.random.default_rng(seed)
        self.num_pages = int(need.sum()) + spare_pages + 2
        ids = rng.permutation(self.num_pages)
        self.bt = np.full((len(need), width or max(1, int(need.max()) + spare_pages)), ids[-1], np.int64)
        at = 0
        for b, k in enumerate(need):
            k = min(k, self.bt.shape[1])
            self.bt[b, :k] = ids[at:at + k]
            at += k
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.g = g
        self.k, self.v = (torch.randn(self.num_pages, PAGE, hkv, d, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        self.q_start = np.concatenate([[0], np.cumsum(self.new)])
        self.block_table, self.d_start, self.d_ctx = cuda(self.bt), cuda(self.q_start), cuda(self.ctx)

    def slots(self, b, lo, hi):
        """Rows of the pool seen as [pages * 16, ...] that hold positions lo..hi of sequence b."""
        t = np.arange(lo, hi)
        return cuda(self.bt[b, t // PAGE] * PAGE + t % PAGE, torch.int64)


def attention(q, k, v, ctx, scale):
    """Causal attention of n new rows q [n, Hq, D] over k, v [ctx + n, Hkv, D]: (out, lse, bound of out, bound of lse), all 64 bits.

    The bound of the output: probabilities rounded to bf16 for their product with V, the output rounded once, and fp32 accumulation (under
    one rounding of 2^-22 per 16 keys and per 16 dims, for an accumulator that drops bits).  That of lse: the scores' accumulation and the sum's."""
    n, hq, d = q.shape
    L, hkv = k.shape[:2]
    G = hq // hkv
    out, lse, b_out, b_lse = (torch.empty(n, hq, *s, device=q.device, dtype=F8) for s in ((d,), (), (d,), ()))
    hidden = torch.arange(L, device=q.device) > torch.arange(ctx, ctx + n, device=q.device)[:, None]
    for h in range(hq):
        kk, vv, qq = k[:, h // G].to(F8), v[:, h // G].to(F8), q[:, h].to(F8)
        s = (qq @ kk.t() * scale).masked_fill_(hidden, -math.inf)
        off = ((qq.abs() @ kk.abs().t()).masked_fill_(hidden, 0).amax(1) * abs(scale) + 1) * (d / 16 + 4) * 2.0 ** -22
        p = torch.softmax(s, 1)
        out[:, h], lse[:, h] = p @ vv, torch.logsumexp(s, 1)
        mass = p @ vv.abs()
        b_out[:, h] = BF16_HALF * 1.01 * (mass + out[:, h].abs()) + mass * (2 * off[:, None] + L / 16 * 2.0 ** -22)
        b_lse[:, h] = off + (L / 32 + 64) * 2.0 ** -22 + lse[:, h].abs() * 2.0 ** -22
    return out, lse, b_out, b_lse


def likelihoods(x, tok, top):
    """Rows x [n, V] of logits in any type, tokens [n]: dict of 64-bit values, and their bounds.

    Bound: fp32 sums whose longest chain is V / 256 additions of a thread and some 40 behind it; an exponential is off by 2^-22 and by its
    argument's rounding, 2^-23 |d|; logf by 2 units, and two roundings of the result."""
    x = x.to(F8)
    V = x.shape[1]
    m = x.amax(1, keepdim=True)
    d = x - m
    e = d.exp()
    Z = e.sum(1)
    p = e / Z[:, None]
    pd = torch.where(e > 0, p * d, 0)
    rel = (V / 256 + 40) * 2.0 ** -24 + 2.0 ** -22 + pd.abs().sum(1) * 2.0 ** -22
    second = torch.where(e > 0, p * d * d, 0).sum(1)
    off = rel + 3 * Z.log().abs() * 2.0 ** -23
    ref, bound = {}, {}
    if tok is not None:
        ref["logprobs"] = d.gather(1, tok[:, None].long())[:, 0] - Z.log()
        bound["logprobs"] = off + 3 * ref["logprobs"].abs() * 2.0 ** -24 + d.gather(1, tok[:, None].long())[:, 0].abs() * 2.0 ** -24
    ref["entropy"] = Z.log() - pd.sum(1)
    bound["entropy"] = off + 2 * rel * pd.abs().sum(1) + second * 2.0 ** -22 + 3 * ref["entropy"].abs() * 2.0 ** -24
    if top:
        order = torch.argsort(x, dim=1, descending=True, stable=True)[:, :top]
        ref["top_ids"] = order
        ref["top_logprobs"] = d.gather(1, order) - Z.log()[:, None]
        bound["top_logprobs"] = off[:, None] + 5 * ref["top_logprobs"].abs() * 2.0 ** -24
    return ref, bound
