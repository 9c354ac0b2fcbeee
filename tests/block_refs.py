"""Plain references of page assignment, slot maps, block summaries, selection and attention over selected blocks."""
import math

import numpy as np
import torch

from tests.operator_refs import BF16_HALF, F8, PAGE, cuda


def assign(want, table, held, free, n_free):
    """One call on host arrays, in place; returns (n_free, sequences left alone for want of pages)."""
    B, M = table.shape
    target = [-(-int(w) // PAGE) for w in want]
    alone = {b for b in range(B) if target[b] > M}
    given = [int(table[b, c]) for b in range(B) if b not in alone for c in range(target[b], held[b])]
    avail = given + [int(free[n_free - 1 - i]) for i in range(n_free)]
    at = 0
    asked = 0
    for b in range(B):
        if b in alone:
            continue
        if target[b] > held[b]:
            asked += target[b] - held[b]
            if asked > len(avail):
                alone.add(b)
                continue
            for c in range(held[b], target[b]):
                table[b, c] = avail[at]
                at += 1
        held[b] = target[b]
    left = avail[at:]
    free[:len(left)] = left[::-1]
    return len(left), alone


def summary(keys):
    """keys [n, heads, D] of a block's tokens: (k_mean int, k_scale), 64 bits.  The mean is a quotient (a mean by multiplication with 1 / n, which has no exact form
    for n = 5, say, puts numbers half way between two steps on the other side)."""
    s = keys.to(F8).sum(0)
    m = s / torch.full_like(s, keys.shape[0])
    top = m.abs().amax(-1, keepdim=True)
    return torch.round(127 * m / top.clamp(min=1e-30)).long(), (top / 127)[..., 0]


def whole_queries(x):
    """The 8-bit whole numbers of queries that vote together."""
    top = torch.clamp(x.float().abs().max(), min=1e-30)
    return torch.round(x.float() * (torch.full_like(top, 127.0) / top)).long()


def select(q, mean, scale, K, n_first, n_last):
    """q [votes, D], mean int8 [nb, D], scale [nb] of one kv head: the chosen blocks, a list."""
    nb = mean.shape[0]
    if q.shape[0] == 0:
        return []
    if nb <= K:
        return list(range(nb))
    dot = (whole_queries(q).to(F8) @ mean.to(F8).t()).amax(0)
    s = (dot.float() * scale).cpu().numpy()
    forced = set(range(n_first)) | set(range(nb - n_last, nb))
    key = lambda j: (-math.inf if math.isnan(s[j]) else -float(s[j]), not math.isnan(s[j]), j)
    rest = sorted((j for j in range(nb) if j not in forced), key=key)
    return sorted(forced | set(rest[:K - len(forced)]))


def positions(blocks, ctx, block):
    return np.concatenate([np.arange(j * block, min((j + 1) * block, ctx)) for j in blocks] + [np.zeros(0, np.int64)]).astype(np.int64)


def masked_attention(q, k, v, visible, scale):
    """q [n, G, D] of one kv head over k, v [L, D], visible [n, L]: (out, lse, bounds) in 64 bits; the bounds as in operator_refs.attention.  A row that
    sees nothing is zero in both."""
    n, G, d = q.shape
    L = k.shape[0]
    out, lse = torch.zeros(n, G, d, device=q.device, dtype=F8), torch.zeros(n, G, device=q.device, dtype=F8)
    b_out, b_lse = torch.zeros_like(out), torch.zeros_like(lse)
    kk, vv = k.to(F8), v.to(F8)
    some = visible.any(1)
    for g in range(G):
        qq = q[:, g].to(F8)
        s = (qq @ kk.t() * scale).masked_fill(~visible, -math.inf)
        off = ((qq.abs() @ kk.abs().t()).masked_fill(~visible, 0).amax(1) * abs(scale) + 1) * (d / 16 + 4) * 2.0 ** -22
        p = torch.where(some[:, None], torch.softmax(s, 1), 0)
        out[:, g] = p @ vv
        lse[:, g] = torch.where(some, torch.logsumexp(s, 1), 0)
        mass = p @ vv.abs()
        b_out[:, g] = BF16_HALF * 1.01 * (mass + out[:, g].abs()) + mass * (2 * off[:, None] + L / 16 * 2.0 ** -22)
        b_lse[:, g] = off + (L / 32 + 64) * 2.0 ** -22 + lse[:, g].abs() * 2.0 ** -22
    return out, lse, b_out, b_lse


def random_lists(ctx, hkv, K, block, seed):
    """Lists as selection leaves them: any blocks, the newest one last."""
    rng = np.random.default_rng(seed)
    out = np.full((len(ctx), hkv, K), -1, np.int64)
    for b, c in enumerate(ctx):
        nb = -(-int(c) // block)
        for h in range(hkv):
            out[b, h, :min(nb, K)] = np.arange(nb) if nb <= K else np.append(np.sort(rng.choice(nb - 1, K - 1, replace=False)), nb - 1)
    return out


def random_trees(B, T, n, seed):
    """Visible [B, T, T] of random trees, and the mask words int32 [B, T, W] on the GPU."""
    rng = np.random.default_rng(seed)
    vis = np.zeros((B, T, T), bool)
    for b in range(B):
        for i in range(int(n[b])):
            if i:
                vis[b, i] = vis[b, rng.integers(0, i)]
            vis[b, i, i] = True
    return vis, mask_words(vis)


def mask_words(vis):
    B, T, _ = vis.shape
    W = (T + 31) // 32
    full = np.zeros((B, T, W * 32), bool)
    full[..., :T] = vis
    return cuda(np.packbits(full.reshape(B, T, W, 32), axis=-1, bitorder="little").view(np.uint32).reshape(B, T, W).view(np.int32))
