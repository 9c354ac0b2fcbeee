"""Performance cases of the operators beside the draft-and-verify step: what a serving program needs to bring a prompt into the paged cache,
to prepare a draft tree for its verification pass, and to say how likely the emitted tokens were.

Operators and the kinds of cases that call them:
  attn      attention of each sequence's chunk of new tokens over its paged cache, which holds the chunk's own keys (cb_chunk_attn)
  append    norm of queries and keys per head, rotation by position, keys and values into the pages (cb_chunk_append)
  tree      the same norm and rotation for the nodes of a draft tree, into the tensors that tree attention reads (cb_tree_rope)
  logprobs  log probability of a given token per row of logits, entropy and the best alternatives (cb_logprobs)
  accept    the same for the tokens that acceptance emitted, from the rows of the tree's nodes (cb_accept_logprobs)

Lengths are spread evenly over the stated range and dealt to the sequences by the seed, so that the work of a case does not depend on it.
"""
import math

import numpy as np
import torch

own = False            # True: the framework's kernels; False: the same in elementary operations, in 32 bits, rounded once at the end

DEV = "cuda:0"
PAGE = 16
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------- the cases
def _attn(name, batch, hq, hkv, d, new_lo, new_hi, ctx_lo, ctx_hi):
    return dict(name=name, kind="attn", batch=batch, hq=hq, hkv=hkv, d=d, new_lo=new_lo, new_hi=new_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi)


def _append(name, batch, hq, hkv, d, new_lo, new_hi, ctx_lo, ctx_hi, rot, norm, interleaved):
    return dict(name=name, kind="append", batch=batch, hq=hq, hkv=hkv, d=d, new_lo=new_lo, new_hi=new_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, rot=rot, norm=norm,
                interleaved=interleaved)


def _tree(name, batch, hq, hkv, d, t, ctx_lo, ctx_hi, rot, norm, interleaved, trees):
    return dict(name=name, kind="tree", batch=batch, hq=hq, hkv=hkv, d=d, t=t, ctx_lo=ctx_lo, ctx_hi=ctx_hi, rot=rot, norm=norm, interleaved=interleaved,
                trees=trees)


def _logprobs(name, rows, vocab, dtype, top, masked):
    return dict(name=name, kind="logprobs", rows=rows, vocab=vocab, dtype=dtype, top=top, masked=masked)


def _accept(name, batch, t, depth, vocab, dtype, top):
    return dict(name=name, kind="accept", batch=batch, t=t, depth=depth, vocab=vocab, dtype=dtype, top=top)


def listed():
    return [
        # one user's chat without a draft: a single new token on a 7B-shaped model, every layer calls this once per token
        _attn("attn_token_b1_4k_mha", 1, 32, 32, 128, 1, 1, 4096, 4096),
        # a server's batch of single tokens over ragged contexts, grouped heads
        _attn("attn_token_b64_ragged_gqa4", 64, 32, 8, 128, 1, 1, 120, 8192),
        # prompts cut into chunks among single tokens, as a scheduler mixes them; head_dim 64, lengths that are no round numbers
        _attn("attn_mixed_b24_d64", 24, 16, 4, 64, 0, 509, 3, 5003),
        # four prompts of a server's batch, nothing cached yet
        _attn("attn_prompts_b4_gqa4", 4, 32, 8, 128, 777, 2048, 0, 0),
        # a whole prompt of 8 k tokens on a 70B-shaped model: the largest call
        _attn("attn_prompt_8k_gqa8", 1, 64, 8, 128, 8192, 8192, 0, 0),
        # the new tokens of a batch of 32 single-token steps: the smallest call, its latency counts
        _append("append_token_b32_gqa4", 32, 32, 8, 128, 1, 1, 100, 1500, 128, True, False),
        # the same prompt of 8 k tokens
        _append("append_prompt_8k_gqa8", 1, 64, 8, 128, 8192, 8192, 0, 0, 128, True, False),
        # the trees of a verification pass at batch 32
        _tree("tree_b32_t64_gqa4", 32, 32, 8, 128, 64, 1024, 8192, 128, True, False, "full"),
        # uneven trees of a small batch, half of a 64-dim head rotated in neighbouring pairs, no norm
        _tree("tree_b13_t61_d64_half", 13, 16, 4, 64, 61, 777, 5003, 32, False, True, "ragged"),
        # scoring a prompt: log probabilities and entropy of 2 k rows over a 128 k vocabulary
        _logprobs("logprobs_prompt_2k_v128k_bf16", 2048, 128256, "bf16", 0, False),
        # a batch of sampled tokens with 20 alternatives each, an odd vocabulary, some ids forbidden
        _logprobs("logprobs_b300_v50k_f32_top20", 300, 50257, "f32", 20, True),
        # the tokens that one sequence's acceptance emitted, with five alternatives
        _accept("accept_b1_t64_v32k_bf16_top5", 1, 64, 8, 32000, "bf16", 5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(8, 8), (32, 32), (40, 40), (32, 8), (64, 8), (16, 4), (28, 4)]


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "tree", "logprobs", "logprobs", "accept"])
    hq, hkv = rng.choice(_HEADS)
    d = rng.choice([64, 128, 128])
    rot = rng.choice([d, d, d // 2])
    norm, inter = rng.random() < 0.6, rng.random() < 0.4
    if kind == "attn":
        shape = rng.choice(["token", "mixed", "prompt"])
        batch = _log_int(rng, 1, 96) if shape != "prompt" else _log_int(rng, 1, 8)
        new_hi = 1 if shape == "token" else (_log_int(rng, 2, 700) if shape == "mixed" else _log_int(rng, 100, 6000))
        new_lo = (1 if shape == "token" else rng.randint(0, 1)) if shape != "prompt" else max(1, int(new_hi * rng.uniform(0.2, 1.0)))
        room = min(20000, int(2e9 / (batch * hkv * d * 4)), int(2.5e9 / (batch * hq * new_hi)) - new_hi, int(8e11 / (4.0 * batch * hq * d * new_hi)) - new_hi)
        if room < 1:                                                   # the largest that costs no more than the largest listed case
            batch, new_hi, room = 1, min(new_hi, 2000), 2000
            new_lo = min(new_lo, new_hi)
        ctx_hi = _log_int(rng, 1, room) if rng.random() < 0.8 else 0
        ctx_lo = int(ctx_hi * rng.uniform(0.0, 1.0))
        c = _attn("", batch, hq, hkv, d, new_lo, new_hi, ctx_lo, ctx_hi)
    elif kind == "append":
        batch = _log_int(rng, 1, 96)
        new_hi = _log_int(rng, 1, max(1, min(8192, 16384 // batch)))
        new_lo = rng.randint(0, new_hi) if batch > 1 else new_hi
        ctx_hi = rng.randint(0, 1500)
        c = _append("", batch, hq, hkv, d, new_lo, new_hi, rng.randint(0, ctx_hi), ctx_hi, rot, norm, inter)
    elif kind == "tree":
        ctx_hi = _log_int(rng, 1, 9000)
        c = _tree("", _log_int(rng, 1, 96), hq, hkv, d, _log_int(rng, 2, 128), int(ctx_hi * rng.random()), ctx_hi, rot, norm, inter, rng.choice(["full", "ragged"]))
    else:
        vocab = rng.choice([32000, 128256, 151936, 50257, _log_int(rng, 1000, 150000)])
        dtype = rng.choice(["f32", "bf16"])
        top = rng.choice([0, 1, 5, 20, rng.randint(1, 32)])
        if kind == "logprobs":
            rows = _log_int(rng, 1, max(1, min(2048, int((2.4e8 if top == 0 else 6e7) / vocab))))
            c = _logprobs("", rows, vocab, dtype, top, rng.random() < 0.3)
        else:
            t = _log_int(rng, 8, 128)
            batch = _log_int(rng, 1, 48)
            while batch * t * vocab > 1.2e8:
                batch, t = (batch // 2, t) if batch > 1 else (1, max(8, t // 2))
            c = _accept("", batch, t, rng.randint(2, 7), vocab, dtype, top)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------- inputs
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 64 + salt)
    return g


def _spread(lo, hi, n):
    """n whole numbers spread evenly over [lo, hi]; the largest is hi."""
    return np.array([hi], np.int64) if n == 1 else np.round(np.linspace(lo, hi, n)).astype(np.int64)


def _lengths(case):
    """New tokens and cached tokens of each sequence, paired the same way for every seed."""
    B = case["batch"]
    return _spread(case["new_lo"], case["new_hi"], B), _spread(case["ctx_lo"], case["ctx_hi"], B)[np.random.RandomState(5).permutation(B)]


def _dealt(case, seed):
    p = np.random.RandomState(seed % (1 << 31)).permutation(case["batch"])
    new, ctx = _lengths(case)
    return new[p], ctx[p]


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def _normal(shape, g, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16).mul_(scale)


def _pages(case, new, ctx, seed):
    """Block table of shuffled pages, as an allocator leaves them, and the number of pages."""
    need = -(-(new + ctx) // PAGE)
    total = int(need.sum()) + 3
    ids = np.random.RandomState((seed + 9) % (1 << 31)).permutation(total)
    bt = np.zeros((case["batch"], int(need.max()) + 1), np.int64)
    at = 0
    for b, k in enumerate(need):
        bt[b, :k] = ids[at:at + k]
        at += k
    return _dev(bt), total


def _rope_table(positions, rot):
    """[positions, rot]: cosines, then sines, of position times 10000^(-2 i / rot); angles in 64 bits."""
    ang = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    return torch.cat((ang.cos(), ang.sin()), 1).float()


def _logits(shape, dtype, g):
    """Logits as a head emits them: a spread of a few units, some rows sure of a token and some not."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)
    x.mul_(torch.rand(shape[:-1], generator=g, device=DEV)[..., None].mul_(3.0).add_(0.5))
    return x if dtype == "f32" else x.to(torch.bfloat16)


def _context(case, **kw):
    """The library's context that a user's program keeps."""
    from paper_2511_21699_b200 import Cacheback
    shape = dict(n_q_heads=case.get("hq", 1), n_kv_heads=case.get("hkv", 1), head_dim=case.get("d", 64), vocab=case.get("vocab", 1),
                 max_nodes=case.get("t", 1), max_depth=case.get("depth", 8))
    return Cacheback(case.get("batch", 1), 1, 1, 1, 1, crt=0, **{**shape, **kw})


def prepare(case, seed):
    kind, s = case["kind"], dict(case)
    if own:
        s["cb"] = _context(case)
    if kind in ("attn", "append"):
        new, ctx = _dealt(case, seed)
        n_rows = int(new.sum())
        s["q_start"], s["ctx_len"] = _dev(np.concatenate([[0], np.cumsum(new)])), _dev(ctx)
        s["new_max"], s["len_max"] = int(new.max()), max(1, int((new + ctx).max()))
        s["block_table"], pages = _pages(case, new, ctx, seed)
        s["k_pool"] = _normal((pages, PAGE, case["hkv"], case["d"]), _gen(seed, 1))
        s["v_pool"] = _normal((pages, PAGE, case["hkv"], case["d"]), _gen(seed, 2))
        if kind == "attn":
            s["q"] = _normal((n_rows, case["hq"], case["d"]), _gen(seed, 3), 1.5)
            s["out"] = torch.zeros_like(s["q"])
            s["lse"] = torch.zeros(n_rows, case["hq"], device=DEV)
            return s
    if kind == "tree":
        B, T = case["batch"], case["t"]
        deal = np.random.RandomState((seed + 1) % (1 << 31))
        n = np.full(B, T) if case["trees"] == "full" else deal.permutation(_spread(1, T, B) if B > 1 else np.array([max(1, T // 3)]))
        depth = np.minimum(np.floor(np.sqrt(np.arange(T))), 24)[None].repeat(B, 0)                 # a tree that widens as it grows
        depth[np.arange(T)[None] >= n[:, None]] = -1
        ctx = deal.permutation(_spread(case["ctx_lo"], case["ctx_hi"], B))
        s["tree"] = dict(depth=_dev(depth), n_nodes=_dev(n))
        s["ctx_len"], n_rows = _dev(ctx), B * T
        s["len_max"] = int(ctx.max()) + 25
    if kind in ("append", "tree"):
        # the model's projection of a row: its query heads, then its key heads, then its value heads
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        qkv = _normal((n_rows, hq + 2 * hkv, d), _gen(seed, 4), 1.5)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["rope"] = _rope_table(max(4096, s["len_max"]), case["rot"])
        s["q_norm"] = _normal((d,), _gen(seed, 5), 0.2).add_(1.0) if case["norm"] else None
        s["k_norm"] = _normal((d,), _gen(seed, 6), 0.2).add_(1.0) if case["norm"] else None
        lead = (case["batch"], case["t"]) if kind == "tree" else (n_rows,)
        s["q_out"] = torch.zeros(*lead, hq, d, device=DEV, dtype=torch.bfloat16)
        if kind == "tree":
            s["k_out"], s["v_out"] = (torch.zeros(*lead, hkv, d, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        return s
    if kind == "logprobs":
        g = _gen(seed, 7)
        x = s["logits"] = _logits((case["rows"], case["vocab"]), case["dtype"], g)
        tok = torch.randint(case["vocab"], (case["rows"],), generator=g, device=DEV)
        if case["masked"]:                                             # ids that a grammar forbids
            x[:, torch.randint(case["vocab"], (case["vocab"] // 4,), generator=g, device=DEV)] = -math.inf
            tok = torch.where(x.gather(1, tok[:, None])[:, 0].isinf(), x.argmax(1), tok)
        s["tokens"] = torch.where(torch.rand(case["rows"], generator=g, device=DEV) < 0.6, x.argmax(1), tok).to(torch.int32)
        s["n_out"] = (case["rows"],)
    else:
        B, T, Dm = case["batch"], case["t"], case["depth"]
        x = s["logits"] = _logits((B, T, case["vocab"]), case["dtype"], _gen(seed, 7))
        rng = np.random.RandomState((seed + 2) % (1 << 31))
        m = rng.permutation(_spread(0, Dm, B))
        nodes = np.full((B, Dm), -1)
        for b in range(B):
            nodes[b, :m[b]] = np.sort(rng.choice(np.arange(1, T), m[b], replace=False))
        s["n_accept"], s["accept_nodes"] = _dev(m), _dev(nodes)
        rows = np.arange(B)[:, None] * T + np.concatenate([np.zeros((B, 1), int), nodes.clip(0)], 1)
        best = x.view(B * T, -1)[_dev(rows, torch.int64)].argmax(-1).to(torch.int32)
        s["out_tokens"] = torch.where(_dev(np.arange(Dm + 1)[None] <= m[:, None], torch.bool), best, -1)
        s["n_out"] = (B, Dm + 1)
    s["res"] = dict(logprobs=torch.zeros(s["n_out"], device=DEV), entropy=torch.zeros(s["n_out"], device=DEV))
    if case["top"]:
        s["res"]["top_ids"] = torch.zeros(*s["n_out"], case["top"], device=DEV, dtype=torch.int32)
        s["res"]["top_logprobs"] = torch.zeros(*s["n_out"], case["top"], device=DEV)
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms
def _plain_attn(s):
    q, B, n, L = s["q"], s["batch"], s["new_max"], s["len_max"]
    N, Hq, D = q.shape
    Hkv = s["hkv"]
    G = Hq // Hkv
    first, ctx = s["q_start"][:-1].long(), s["ctx_len"].long()
    i, j = torch.arange(n, device=DEV), torch.arange(L, device=DEV)
    page, slot = s["block_table"].long()[:, j // PAGE], j % PAGE
    K, V = (s[x][page, slot].float().permute(0, 2, 1, 3) for x in ("k_pool", "v_pool"))          # [B, Hkv, L, D]
    Q = q[(first[:, None] + i).clamp_(max=N - 1)].float().view(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    S = torch.matmul(Q, K.transpose(2, 3)).mul_(D ** -0.5).view(B, Hkv, G, n, L)
    S.masked_fill_((j > ctx[:, None, None] + i[:, None])[:, None, None], -math.inf)
    m = S.amax(-1, keepdim=True)
    P = S.sub_(m).exp_()
    Z = P.sum(-1, keepdim=True)
    O = torch.matmul(P.view(B, Hkv, G * n, L), V).view(B, Hkv, G, n, D).div_(Z)
    lse = (m + Z.log())[..., 0]
    r = torch.arange(N, device=DEV)
    b = torch.searchsorted(s["q_start"].long(), r, right=True) - 1
    return O[b, :, :, r - first[b]].reshape(N, Hq, D).to(q.dtype), lse[b, :, :, r - first[b]].reshape(N, Hq)


def _plain_rope(s, x, weight, pos):
    x, R = x.float(), s["rot"]
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    c, sn = s["rope"][pos, None, :R // 2], s["rope"][pos, None, R // 2:]
    if s["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y = torch.stack((a * c - b * sn, b * c + a * sn), -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y = torch.cat((a * c - b * sn, b * c + a * sn), -1)
    return torch.cat((y, x[..., R:]), -1).to(torch.bfloat16)


def _plain_append(s):
    r = torch.arange(s["q"].shape[0], device=DEV)
    b = torch.searchsorted(s["q_start"].long(), r, right=True) - 1
    pos = s["ctx_len"].long()[b] + r - s["q_start"].long()[b]
    page, slot = s["block_table"].long()[b, pos // PAGE], pos % PAGE
    s["k_pool"][page, slot] = _plain_rope(s, s["k"], s["k_norm"], pos)
    s["v_pool"][page, slot] = s["v"]
    return _plain_rope(s, s["q"], s["q_norm"], pos), s["k_pool"], s["v_pool"]


def _plain_tree(s):
    B, T = s["batch"], s["t"]
    valid = (torch.arange(T, device=DEV) < s["tree"]["n_nodes"][:, None]).view(-1, 1, 1)
    pos = (s["ctx_len"].long()[:, None] + s["tree"]["depth"]).clamp_(min=0).view(-1)
    got = (_plain_rope(s, s["q"], s["q_norm"], pos), _plain_rope(s, s["k"], s["k_norm"], pos), s["v"])
    return tuple(torch.where(valid, x, 0).view(B, T, *x.shape[1:]) for x in got)


def _plain_logprobs(x, tok, top):
    x = x.float()
    d = x - x.amax(-1, keepdim=True)
    e = d.exp()
    Z = e.sum(-1)
    ent = Z.log() - torch.where(e > 0, e * d, 0).sum(-1) / Z
    res = dict(logprobs=d.gather(1, tok.long()[:, None])[:, 0] - Z.log(), entropy=ent)
    if top:
        v, i = torch.sort(d, dim=-1, descending=True, stable=True)     # equal values: the lowest id first
        res["top_ids"], res["top_logprobs"] = i[:, :top].to(torch.int32), v[:, :top] - Z.log()[:, None]
    return res


def _plain_accept(s):
    B, T = s["batch"], s["t"]
    node = torch.cat((torch.zeros(B, 1, device=DEV, dtype=torch.int32), s["accept_nodes"]), 1).long()
    rows = torch.arange(B, device=DEV)[:, None] * T + node.clamp(min=0)
    tok, valid = s["out_tokens"].view(-1), (s["out_tokens"] >= 0).view(-1)
    res = _plain_logprobs(s["logits"].view(B * T, -1)[rows.view(-1)], tok.clamp(min=0), s["top"])
    res = {k: torch.where(valid[:, None] if v.dim() > 1 else valid, v, -1 if k == "top_ids" else 0.0) for k, v in res.items()}
    return {k: v.view(B, -1, *v.shape[1:]) for k, v in res.items()}


def run(s):
    kind = s["kind"]
    if own:
        cb = s["cb"]
        if kind == "attn":
            cb.cb_chunk_attn(s["q"], s["k_pool"], s["v_pool"], s["block_table"], s["q_start"], s["ctx_len"], out=s["out"], lse=s["lse"],
                             max_chunk=s["new_max"], max_ctx=s["len_max"])
            return s["out"], s["lse"]
        if kind == "append":
            cb.cb_chunk_append(s["q"], s["k"], s["v"], s["q_start"], s["ctx_len"], s["k_pool"], s["v_pool"], s["block_table"], rope=s["rope"],
                               q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS, interleaved=s["interleaved"], q_out=s["q_out"])
            return s["q_out"], s["k_pool"], s["v_pool"]
        if kind == "tree":
            return cb.cb_tree_rope(s["q"], s["k"], s["v"], s["tree"], s["ctx_len"], rope=s["rope"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS,
                                   interleaved=s["interleaved"], q_out=s["q_out"], k_out=s["k_out"], v_out=s["v_out"])
        if kind == "logprobs":
            return cb.cb_logprobs(s["logits"], s["tokens"], top_k=s["top"], res=s["res"])
        return cb.cb_accept_logprobs(s["logits"], s, top_k=s["top"], res=s["res"])
    if kind == "attn":
        return _plain_attn(s)
    if kind == "append":
        return _plain_append(s)
    if kind == "tree":
        return _plain_tree(s)
    if kind == "logprobs":
        return _plain_logprobs(s["logits"], s["tokens"], s["top"])
    return _plain_accept(s)


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "attn":
        new, ctx = _lengths(case)
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        keys = int(((new + ctx) * (new > 0)).sum())
        seen = int((new * ctx + new * (new + 1) // 2).sum())
        rows = int(new.sum())
        return {"bytes": keys * hkv * d * 4 + rows * hq * (d * 4 + 4) + keys // PAGE * 4, "flops": 4 * hq * d * seen}
    if kind in ("append", "tree"):
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        if kind == "append":
            rows = out = int(_lengths(case)[0].sum())
        else:
            B, T = case["batch"], case["t"]
            rows = B * T if case["trees"] == "full" else (int(_spread(1, T, B).sum()) if B > 1 else max(1, T // 3))
            out = B * T
        return {"bytes": (rows + out) * (hq + 2 * hkv) * d * 2 + rows * (case["rot"] * 4 + 4), "flops": rows * (hq + hkv) * (3 * case["rot"] + (4 * d if case["norm"] else 0))}
    rows = case["rows"] if kind == "logprobs" else int((_spread(0, case["depth"], case["batch"]) + 1).sum())
    size = 4 if case["dtype"] == "f32" else 2
    return {"bytes": rows * (case["vocab"] * size + 12 + 8 * case["top"]), "flops": 5 * rows * case["vocab"]}


# ---------------------------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    kind, s = case["kind"], prepare(case, seed)
    f8 = torch.float64
    if kind == "attn":
        q, scale = s["q"], 1.0 / math.sqrt(case["d"])
        out, lse = torch.empty(q.shape, device=DEV, dtype=f8), torch.empty(q.shape[:2], device=DEV, dtype=f8)
        start, G = s["q_start"].tolist(), case["hq"] // case["hkv"]
        for b, c in enumerate(s["ctx_len"].tolist()):
            lo, hi = start[b], start[b + 1]
            if hi == lo:
                continue
            t = torch.arange(c + hi - lo, device=DEV)
            at = s["block_table"][b].long()[t // PAGE] * PAGE + t % PAGE
            hidden = t > torch.arange(c, c + hi - lo, device=DEV)[:, None]
            for kh in range(case["hkv"]):
                k, v = (s[x].view(-1, case["hkv"], case["d"])[at, kh].to(f8) for x in ("k_pool", "v_pool"))
                for h in range(kh * G, kh * G + G):
                    z = q[lo:hi, h].to(f8) @ k.t() * scale
                    z[hidden] = -math.inf
                    lse[lo:hi, h] = torch.logsumexp(z, 1)
                    out[lo:hi, h] = torch.softmax(z, 1) @ v
        return out, lse
    if kind in ("append", "tree"):
        hq, hkv, d, R = case["hq"], case["hkv"], case["d"], case["rot"]
        n_rows = s["q"].shape[0]
        if kind == "append":
            first, ctx = s["q_start"].cpu().numpy(), s["ctx_len"].cpu().numpy()
            pos = np.concatenate([ctx[b] + np.arange(first[b + 1] - first[b]) for b in range(len(ctx))]).astype(np.int64)
        else:
            pos = (s["ctx_len"].cpu().numpy()[:, None] + s["tree"]["depth"].cpu().numpy()).reshape(-1).astype(np.int64)
        pos = _dev(pos.clip(0), torch.int64)
        turn = torch.complex(s["rope"][pos, :R // 2].to(f8), s["rope"][pos, R // 2:].to(f8))[:, None]

        def turned(x, w):
            y = x.to(f8)
            if w is not None:
                y = y / (y.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * w.to(f8)
            head = y[..., :R]
            pair = head.reshape(*head.shape[:-1], R // 2, 2) if case["interleaved"] else head.reshape(*head.shape[:-1], 2, R // 2).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            return torch.cat(((z if case["interleaved"] else z.transpose(-1, -2)).reshape(head.shape), y[..., R:]), -1)

        qo, ko, vo = turned(s["q"], s["q_norm"]), turned(s["k"], s["k_norm"]), s["v"].to(f8)
        if kind == "tree":
            T = case["t"]
            dead = torch.arange(T, device=DEV)[None] >= s["tree"]["n_nodes"][:, None]
            res = [x.reshape(case["batch"], T, -1, d).clone() for x in (qo, ko, vo)]
            for x in res:
                x[dead] = 0
            return tuple(res)
        kp, vp, bt = s["k_pool"].to(f8), s["v_pool"].to(f8), s["block_table"].long()
        seq = _dev(np.repeat(np.arange(len(ctx)), np.diff(first)), torch.int64)
        at = bt[seq, pos // PAGE] * PAGE + pos % PAGE
        kp.view(-1, hkv, d)[at] = ko
        vp.view(-1, hkv, d)[at] = vo
        return qo, kp, vp
    V, top = case["vocab"], case["top"]
    x = s["logits"].reshape(-1, V)
    if kind == "logprobs":
        rows, tok = np.arange(case["rows"]), s["tokens"].cpu().numpy()
    else:
        nodes = s["accept_nodes"].cpu().numpy()
        rows = (np.arange(case["batch"])[:, None] * case["t"] + np.concatenate([np.zeros((case["batch"], 1), int), nodes], 1)).reshape(-1)
        tok = s["out_tokens"].cpu().numpy().reshape(-1)
    n = len(rows)
    lp, ent = torch.zeros(n, device=DEV, dtype=f8), torch.zeros(n, device=DEV, dtype=f8)
    ids, alt = torch.full((n, max(top, 1)), -1, device=DEV, dtype=torch.int32), torch.zeros(n, max(top, 1), device=DEV, dtype=f8)
    live = np.nonzero(tok >= 0)[0]
    for k in range(0, len(live), 256):
        w = live[k:k + 256]
        y = torch.log_softmax(x[_dev(rows[w], torch.int64)].to(f8), -1)
        wd = _dev(w, torch.int64)
        lp[wd] = y[torch.arange(len(w), device=DEV), _dev(tok[w], torch.int64)]
        ent[wd] = torch.special.entr(y.exp()).sum(-1)
        if top:
            order = torch.argsort(x[_dev(rows[w], torch.int64)].to(f8), dim=-1, descending=True, stable=True)[:, :top]
            ids[wd], alt[wd] = order.to(torch.int32), y.gather(1, order)
    shape = s["n_out"]
    res = dict(logprobs=lp.view(shape), entropy=ent.view(shape))
    if top:
        res["top_ids"], res["top_logprobs"] = ids.view(*shape, top), alt.view(*shape, top)
    return res
