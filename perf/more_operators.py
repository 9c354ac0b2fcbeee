"""Performance cases of the operators that keep a paged cache and attend to a part of it: block tables and slot maps made on the GPU from the
sequences' lengths, and attention over the blocks of a long context that a cheap score selects.

Operators and the kinds of cases that call them:
  pages    pages given to the sequences that grow and taken back from those that shrink (cb_pages_assign)
  slots    sequence, position and cache slot of every row of a packed batch (cb_slot_map)
  summary  the mean key of every block that new tokens touch, in 8 bits (cb_block_summary)
  select   the blocks that a chunk's or a tree's queries score highest, per sequence and kv head (cb_block_select)
  attn     attention of a chunk over the selected blocks and itself (cb_block_attn)
  tree     the same of a draft tree's nodes (cb_block_tree_attn)

Lengths are spread evenly over the stated range and dealt to the sequences by the seed, so that the work of a case does not depend on it.
"""
import math

import numpy as np
import torch

own = False            # True: the framework's kernels; False: the same in elementary operations, in 32 bits, rounded once at the end

DEV = "cuda:0"
PAGE = 16


# ---------------------------------------------------------------------------------------------------- the cases
def _pages(name, batch, from_lo, from_hi, grow_lo, grow_hi, tight):
    return dict(name=name, kind="pages", batch=batch, from_lo=from_lo, from_hi=from_hi, grow_lo=grow_lo, grow_hi=grow_hi, tight=tight)


def _slots(name, batch, new_lo, new_hi, ctx_lo, ctx_hi, pad):
    return dict(name=name, kind="slots", batch=batch, new_lo=new_lo, new_hi=new_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, pad=pad)


def _summary(name, batch, hkv, d, block, new_lo, new_hi, ctx_lo, ctx_hi):
    return dict(name=name, kind="summary", batch=batch, hkv=hkv, d=d, block=block, new_lo=new_lo, new_hi=new_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi)


def _sparse(name, kind, batch, hq, hkv, d, block, n_select, new_lo, new_hi, ctx_lo, ctx_hi, tree=False):
    """tree: new_hi is the trees' size cap, new_lo the least number of nodes; else chunks of new_lo to new_hi tokens."""
    return dict(name=name, kind=kind, batch=batch, hq=hq, hkv=hkv, d=d, block=block, n_select=n_select, new_lo=new_lo, new_hi=new_hi, ctx_lo=ctx_lo,
                ctx_hi=ctx_hi, tree=tree)


def listed():
    return [
        # a verification step of 32 sequences: pages for the longest draft, then back to what was there; the smallest call
        _pages("pages_step_b32", 32, 1000, 8000, 9, 9, False),
        # 512 requests admitted at once with up to 8 k tokens each, and finished
        _pages("pages_admit_b512", 512, 0, 0, 100, 8192, False),
        # where a batch of single tokens goes
        _slots("slots_token_b32", 32, 1, 1, 100, 8192, 0),
        # 64 prompts or parts of them, up to 2 k tokens each, in a batch that a graph's fixed size pads
        _slots("slots_prompts_b64", 64, 0, 2048, 0, 5003, 999),
        # a step of 64 single tokens: the block that each one falls into
        _summary("summary_token_b64", 64, 8, 128, 64, 1, 1, 100, 1500),
        # four prompts of up to 16 k tokens
        _summary("summary_prompts_b4", 4, 8, 128, 64, 7777, 16384, 0, 0),
        # single tokens over ragged long contexts, grouped heads
        _sparse("select_token_b64", "select", 64, 32, 8, 128, 64, 32, 1, 1, 1000, 32768),
        # the trees of a verification pass at batch 16 with contexts of 32 k
        _sparse("select_tree_b16", "select", 16, 64, 8, 128, 64, 32, 64, 64, 16000, 32768, tree=True),
        # one user's token in a long conversation: latency counts
        _sparse("attn_token_b1", "attn", 1, 32, 8, 128, 64, 32, 1, 1, 32000, 32000),
        # a server's batch of single tokens
        _sparse("attn_token_b64", "attn", 64, 32, 8, 128, 64, 32, 1, 1, 1000, 32768),
        # parts of prompts against what of their long contexts matters
        _sparse("attn_chunk_b8", "attn", 8, 64, 8, 128, 64, 32, 129, 256, 3001, 32768),
        # the trees of a verification pass, 64 nodes each
        _sparse("tree_b16_t64", "tree", 16, 64, 8, 128, 64, 32, 64, 64, 16000, 32768, tree=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(8, 8), (32, 32), (40, 40), (32, 8), (64, 8), (16, 4), (28, 4), (16, 1)]


def draw(rng):
    kind = rng.choice(["pages", "slots", "summary", "select", "select", "attn", "attn", "attn", "tree"])
    hq, hkv = rng.choice(_HEADS)
    d = rng.choice([64, 128, 128])
    block = rng.choice([16, 32, 64, 64, 128])
    if kind == "pages":
        batch = _log_int(rng, 1, 512)
        from_hi = rng.choice([0, _log_int(rng, 1, 8000)])
        grow_hi = _log_int(rng, 1, 8192)
        c = _pages("", batch, int(from_hi * rng.random()), from_hi, rng.randint(0, grow_hi), grow_hi, rng.random() < 0.3)
    elif kind == "slots":
        batch = _log_int(rng, 1, 300)
        new_hi = _log_int(rng, 1, min(8192, max(2, 65536 // batch)))
        ctx_hi = _log_int(rng, 1, 30000)
        c = _slots("", batch, rng.randint(0, new_hi), new_hi, int(ctx_hi * rng.random()), ctx_hi, rng.choice([0, _log_int(rng, 1, 1000)]))
    elif kind == "summary":
        batch = _log_int(rng, 1, 96)
        new_hi = _log_int(rng, 1, max(1, min(16384, 48000 * 1024 // (batch * hkv * d))))
        ctx_hi = _log_int(rng, 1, min(32000, max(100, 48000 * 1024 // (batch * hkv * d))))
        c = _summary("", batch, hkv, d, block, rng.randint(0, new_hi), new_hi, int(ctx_hi * rng.random()), ctx_hi)
    else:
        tree = kind == "tree" or (kind == "select" and rng.random() < 0.4)
        n_select = rng.randint(3, max(4, min(128, 3000 // block)))
        # (selection has something to leave out)
        ctx_hi = _log_int(rng, 20 if kind != "select" else 2 * n_select * block + 64, 40000)
        batch = _log_int(rng, 1, 64)
        new_hi = _log_int(rng, 2, 128) if tree else (1 if rng.random() < 0.5 else _log_int(rng, 2, 256))
        keys = min(ctx_hi, n_select * block) + new_hi
        # no more pages, selected keys and scores than the largest listed cases have
        while batch > 1 and (batch * ctx_hi * hkv * d > 1.0e9 or batch * keys * hkv * d > 1.3e8 or batch * new_hi * hq * keys > 2.5e8):
            batch = max(1, batch * 3 // 4)
        c = _sparse("", kind, batch, hq, hkv, d, block, n_select, rng.randint(1, new_hi) if new_hi > 1 else 1, new_hi, int(ctx_hi * rng.random()), ctx_hi, tree)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------- inputs
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 64 + salt)
    return g


def _host(seed, salt):
    return np.random.RandomState((seed * 64 + salt) % (1 << 31))


def _spread(lo, hi, n):
    """n whole numbers spread evenly over [lo, hi]; the largest is hi."""
    return np.array([hi], np.int64) if n == 1 else np.round(np.linspace(lo, hi, n)).astype(np.int64)


def _lengths(case):
    """New tokens (or nodes) and cached tokens of each sequence, paired the same way for every seed."""
    B = case["batch"]
    return _spread(case["new_lo"], case["new_hi"], B), _spread(case["ctx_lo"], case["ctx_hi"], B)[np.random.RandomState(5).permutation(B)]


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def _normal(shape, g, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16).mul_(scale)


def _table(tokens, seed, room=1):
    """Block table of shuffled pages, as an allocator leaves them, and the number of pages."""
    need = -(-tokens // PAGE)
    total = int(need.sum()) + 61
    ids = _host(seed, 9).permutation(total)
    bt = np.zeros((len(need), int(need.max()) + room), np.int64)
    at = 0
    for b, k in enumerate(need):
        bt[b, :k] = ids[at:at + k]
        at += k
    return bt, total


def _context(case):
    """The library's context that a user's program keeps."""
    from paper_2511_21699_b200 import Cacheback
    return Cacheback(case["batch"], 1, 1, 1, 1, max_nodes=case["new_hi"] if case.get("tree") else 1, crt=0, max_depth=8, vocab=1,
                     n_q_heads=case.get("hq", case.get("hkv", 1)), n_kv_heads=case.get("hkv", 1), head_dim=case.get("d", 64))


def _page_lengths(case):
    """Tokens before and after a step, paired the same way for every seed."""
    B = case["batch"]
    old = _spread(case["from_lo"], case["from_hi"], B)
    return old, old + _spread(case["grow_lo"], case["grow_hi"], B)[np.random.RandomState(7).permutation(B)]


def _prepare_pages(case, s, seed):
    B, rng = case["batch"], _host(seed, 1)
    deal = rng.permutation(B)
    old, new = (x[deal] for x in _page_lengths(case))
    held, want = -(-old // PAGE), -(-new // PAGE)
    spare = int((want - held).sum())
    spare = max(1, spare * 2 // 3) if case["tight"] else spare + 5
    total = int(held.sum()) + spare
    ids = rng.permutation(total)
    bt = np.full((B, int(want.max()) + 2), -1, np.int64)
    at = 0
    for b, k in enumerate(held):
        bt[b, :k] = ids[at:at + k]
        at += k
    free = np.full(total, -1, np.int64)
    free[:spare] = ids[at:]
    s.update(want=_dev(new), back=_dev(old), held=_dev(held), table=_dev(bt), free=_dev(free), n_free=_dev(np.array([spare])))


def _prepare_tree(case, s, seed, n):
    """Ancestor masks of random trees: a node's parent is one of the few nodes before it."""
    B, T, rng = case["batch"], case["new_hi"], _host(seed, 3)
    parent = np.maximum(0, np.arange(T)[None] - 1 - np.minimum(rng.geometric(0.4, (B, T)), 12))
    W = (T + 31) // 32
    vis = np.zeros((B, T, W * 32), bool)
    vis[:, 0, 0] = True
    for i in range(1, T):
        vis[:, i] = vis[np.arange(B), parent[:, i]]
        vis[:, i, i] = True
    vis &= (np.arange(T)[None] < n[:, None])[..., None]
    bits = np.packbits(vis.reshape(B, T, W, 32), axis=-1, bitorder="little").view(np.uint32).reshape(B, T, W)
    s["mask"], s["n_nodes"] = _dev(bits.view(np.int32)), _dev(n)


def prepare(case, seed):
    kind, s = case["kind"], dict(case)
    if own:
        s["cb"] = _context(case)
    if kind == "pages":
        _prepare_pages(case, s, seed)
        return s
    deal = _host(seed, 2).permutation(case["batch"])
    new, ctx = (x[deal] for x in _lengths(case))
    s["q_start"], s["ctx_len"] = _dev(np.concatenate([[0], np.cumsum(new)])), _dev(ctx)
    bt, pages = _table(ctx + (0 if case.get("tree") else new), seed)
    s["table"], s["num_pages"] = _dev(bt), pages
    if kind == "slots":
        n = s["n_rows"] = int(new.sum()) + case["pad"]
        s["res"] = dict(slots=torch.zeros(n, device=DEV, dtype=torch.int64), positions=torch.zeros(n, device=DEV, dtype=torch.int32),
                        seqs=torch.zeros(n, device=DEV, dtype=torch.int32))
        return s
    hkv, d = case["hkv"], case["d"]
    if kind == "summary":
        s["to_len"] = s["ctx_len"] + _dev(new)
        s["k_pool"] = _normal((pages, PAGE, hkv, d), _gen(seed, 1)).add_(_normal((pages, 1, hkv, d), _gen(seed, 2), 0.7))    # what a text's parts have in common
        s["k_mean"], s["k_scale"] = torch.zeros(pages, hkv, d, device=DEV, dtype=torch.int8), torch.zeros(pages, hkv, device=DEV)
        return s
    rows = (case["batch"], case["new_hi"]) if case["tree"] else (int(new.sum()),)
    s["q"] = _normal((*rows, case["hq"], d), _gen(seed, 3), 1.5)
    if case["tree"]:
        _prepare_tree(case, s, seed, new)
    if kind == "select":
        mean = torch.randn(pages, hkv, d, generator=_gen(seed, 4), device=DEV)
        top = mean.abs().amax(-1, keepdim=True)
        s["k_mean"], s["k_scale"] = (mean * (127.0 / top)).round().to(torch.int8), (top[..., 0] * (0.3 / 127.0)).contiguous()
        s["blocks"] = torch.zeros(case["batch"], hkv, case["n_select"], device=DEV, dtype=torch.int32)
        return s
    s["k_pool"], s["v_pool"] = _normal((pages, PAGE, hkv, d), _gen(seed, 1)), _normal((pages, PAGE, hkv, d), _gen(seed, 2))
    if case["tree"]:
        s["k_tree"], s["v_tree"] = _normal((*rows, hkv, d), _gen(seed, 4)), _normal((*rows, hkv, d), _gen(seed, 5))
    # the lists that selection has made: the first block, the newest one, and others between them
    K, rng = case["n_select"], _host(seed, 6)
    blocks = np.full((case["batch"], hkv, K), -1, np.int64)
    for b in range(case["batch"]):
        nb = int(-(-ctx[b] // case["block"]))
        for h in range(hkv):
            if nb <= K:
                blocks[b, h, :nb] = np.arange(nb)
            else:
                blocks[b, h] = np.concatenate([[0], 1 + np.sort(rng.choice(nb - 2, K - 2, replace=False)), [nb - 1]])
    s["blocks"] = _dev(blocks)
    s["out"] = torch.zeros_like(s["q"])
    lse = (case["batch"], case["hq"], case["new_hi"]) if case["tree"] else (rows[0], case["hq"])
    s["lse"] = torch.zeros(lse, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms
def _plain_pages(s, want):
    """avail: the pages given back in order of sequence and place, then the free ones from the top of their stack."""
    table, held, free, n_free = s["table"], s["held"].long(), s["free"], s["n_free"].long()
    B, M = table.shape
    N = free.shape[0]
    target = (want.long() + PAGE - 1) // PAGE
    col = torch.arange(M, device=DEV)
    back = (col >= target[:, None]) & (col < held[:, None])
    n_back = back.sum()
    need = (target - held).clamp(min=0)
    fits = need.cumsum(0) <= n_free + n_back
    got = (col >= held[:, None]) & (col < target[:, None]) & fits[:, None]
    j = torch.arange(N, device=DEV)
    from_top = free[(n_free - 1 - (j - n_back)).clamp(0, N - 1)]
    place = torch.where(back, back.flatten().cumsum(0).view(B, M) - 1, N).flatten()
    given = torch.zeros(N + 1, device=DEV, dtype=table.dtype).scatter_(0, place, table.flatten())[:N]
    avail = torch.where(j < n_back, given, from_top)
    table.copy_(torch.where(got, avail[(got.flatten().cumsum(0).view(B, M) - 1).clamp(0, N - 1)], table))
    total, left = n_free + n_back, n_free + n_back - got.sum()
    free.copy_(torch.where(j < left, avail[(total - 1 - j).clamp(0, N - 1)], free))
    s["held"].copy_(torch.where((need > 0) & ~fits, held, target))
    s["n_free"].copy_(left)


def _plain_slots(s):
    r = torch.arange(s["n_rows"], device=DEV)
    b = torch.searchsorted(s["q_start"].long(), r, right=True) - 1
    in_seq = b < s["batch"]
    b = b.clamp(max=s["batch"] - 1)
    pos = s["ctx_len"].long()[b] + r - s["q_start"].long()[b]
    slot = s["table"].long()[b, torch.where(in_seq, pos // PAGE, 0)] * PAGE + pos % PAGE
    return dict(slots=torch.where(in_seq, slot, -1), positions=torch.where(in_seq, pos, -1).to(torch.int32), seqs=torch.where(in_seq, b, -1).to(torch.int32))


def _plain_summary(s):
    S, M, lo, hi = s["block"], s["table"].shape[1], s["ctx_len"].long(), s["to_len"].long()
    n = (M * PAGE + S - 1) // S
    blk = torch.arange(n, device=DEV)
    hit = (blk >= lo[:, None] // S) & (blk * S < hi[:, None]) & (hi > lo)[:, None]
    b, blk = hit.nonzero(as_tuple=True)
    left = (hi[b] - blk * S).clamp(max=S)
    pos = blk[:, None] * S + torch.arange(S, device=DEV)
    page = s["table"].long()[b[:, None], (pos // PAGE).clamp(max=M - 1)]
    keys = torch.where((pos < hi[b, None])[..., None, None], s["k_pool"][page, pos % PAGE].double(), 0.0)
    mean = keys.sum(1) / left.double()[:, None, None]                  # in 64 bits: means lie next to the steps' borders
    top = mean.abs().amax(-1, keepdim=True)
    at = s["table"].long()[b, blk * S // PAGE]
    s["k_mean"][at] = (mean * 127.0 / top.clamp(min=1e-30)).round().to(torch.int8)
    s["k_scale"][at] = (top / 127.0)[..., 0].float()
    return dict(k_mean=s["k_mean"] * s["k_scale"][..., None], k_scale=s["k_scale"])


def _queries(s, x):
    """[B, rows, ...] of packed rows or of nodes, and which of them there are."""
    if s["tree"]:
        return x, torch.arange(x.shape[1], device=DEV) < s["n_nodes"][:, None]
    first = s["q_start"].long()
    i = torch.arange(s["new_hi"], device=DEV)
    return x[(first[:-1, None] + i).clamp(max=x.shape[0] - 1)], i < (first[1:] - first[:-1])[:, None]


def _plain_select(s):
    B, Hkv, D, S, K = s["batch"], s["hkv"], s["d"], s["block"], s["n_select"]
    q, there = _queries(s, s["q"])
    q = (q.float() * there[..., None, None]).view(B, -1, Hkv, s["hq"] // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    top = q.abs().amax((2, 3), keepdim=True).clamp(min=1e-30)
    q8 = (q * (torch.full_like(top, 127.0) / top)).round()
    nb = (s["ctx_len"].long() + S - 1) // S
    j = torch.arange((s["ctx_hi"] + S - 1) // S, device=DEV)
    page = s["table"].long()[:, j * (S // PAGE)]
    mean, scale = s["k_mean"][page].float().permute(0, 2, 1, 3), s["k_scale"][page].permute(0, 2, 1)
    dot = torch.matmul(q8, mean.transpose(2, 3))                       # whole numbers below 2^21: exact in any order
    rows = there.repeat_interleave(s["hq"] // Hkv, 1)[:, None, :, None]
    score = dot.masked_fill_(~rows, -math.inf).amax(2) * scale
    near = ((j < 1) | (j >= nb[:, None] - 2))[:, None]
    score = torch.where(near, math.inf, score).masked_fill((j >= nb[:, None])[:, None], -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :K]
    order = torch.nn.functional.pad(order, (0, K - order.shape[-1]), value=1 << 30)
    order = torch.where(torch.arange(K, device=DEV) < nb[:, None, None], order, 1 << 30).sort(-1)[0]
    return torch.where(order < 1 << 30, order, -1).to(torch.int32)


def _plain_attn(s):
    B, Hq, Hkv, D, S, K = s["batch"], s["hq"], s["hkv"], s["d"], s["block"], s["n_select"]
    G, ctx = Hq // Hkv, s["ctx_len"].long()
    nb = (ctx + S - 1) // S
    ns = nb.clamp(max=K)
    cached = ctx - (nb - ns) * S                                       # selected keys
    n_new = s["new_hi"]
    v = torch.arange(min(s["ctx_hi"], K * S) + (0 if s["tree"] else n_new), device=DEV)
    listed_at = s["blocks"].long()[:, :, (v // S).clamp(max=K - 1)] * S + v % S
    behind = (nb * S)[:, None] + v - (ns * S)[:, None]
    pos = torch.where(v < (ns * S)[:, None, None], listed_at, behind[:, None]).clamp(0, s["table"].shape[1] * PAGE - 1)
    page = s["table"].long()[torch.arange(B, device=DEV)[:, None, None], pos // PAGE]
    h = torch.arange(Hkv, device=DEV)[:, None]
    keys, vals = (s[x][page, pos % PAGE, h].float() for x in ("k_pool", "v_pool"))
    q, there = _queries(s, s["q"])
    n = q.shape[1]
    q = q.float().view(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    score = torch.matmul(q, keys.transpose(2, 3)).view(B, Hkv, G, n, -1)
    if s["tree"]:
        score.masked_fill_((v >= cached[:, None])[:, None, None, None], -math.inf)
        own_keys = torch.matmul(q, s["k_tree"].float().permute(0, 2, 3, 1)).view(B, Hkv, G, n, n)
        bits = s["mask"].long()[..., torch.arange(n, device=DEV) // 32] >> (torch.arange(n, device=DEV) % 32) & 1
        own_keys.masked_fill_((bits == 0)[:, None, None], -math.inf)
        score = torch.cat((score, own_keys), -1)
        vals = torch.cat((vals, s["v_tree"].float().permute(0, 2, 1, 3)), 2)
    else:
        score.masked_fill_((v > cached[:, None, None] + torch.arange(n, device=DEV)[:, None])[:, None, None], -math.inf)
    score.mul_(D ** -0.5)
    m = score.amax(-1, keepdim=True)
    p = score.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, Hkv, G * n, -1), vals).view(B, Hkv, G, n, D).div_(z)
    lse = (m + z.log())[..., 0]
    if s["tree"]:
        out = torch.where(there[:, None, None, :, None], out, 0.0).permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)
        return out.to(torch.bfloat16), torch.where(there[:, None, None], lse, 0.0).reshape(B, Hq, n)
    N = s["q"].shape[0]
    r = torch.arange(N, device=DEV)
    b = torch.searchsorted(s["q_start"].long(), r, right=True) - 1
    i = r - s["q_start"].long()[b]
    return out[b, :, :, i].reshape(N, Hq, D).to(torch.bfloat16), lse[b, :, :, i].reshape(N, Hq)


def run(s):
    kind = s["kind"]
    if own:
        cb = s["cb"]
        if kind == "pages":
            for want in (s["want"], s["back"]):
                cb.cb_pages_assign(want, s["table"], s["held"], s["free"], s["n_free"])
            return s["table"], s["held"], s["free"], s["n_free"]
        if kind == "slots":
            return cb.cb_slot_map(s["q_start"], s["ctx_len"], s["table"], s["num_pages"], s["n_rows"], res=s["res"])
        if kind == "summary":
            cb.cb_block_summary(s["k_pool"], s["table"], s["ctx_len"], s["to_len"], s["k_mean"], s["k_scale"], block=s["block"])
            return dict(k_mean=s["k_mean"] * s["k_scale"][..., None], k_scale=s["k_scale"])
        if kind == "select":
            rows = dict(n_nodes=s["n_nodes"]) if s["tree"] else dict(q_start=s["q_start"], max_chunk=s["new_hi"])
            return cb.cb_block_select(s["q"], s["k_mean"], s["k_scale"], s["table"], s["ctx_len"], **rows, block=s["block"], n_select=s["n_select"],
                                      n_first=1, n_last=2, max_ctx=s["ctx_hi"], blocks=s["blocks"])
        if kind == "attn":
            cb.cb_block_attn(s["q"], s["k_pool"], s["v_pool"], s["table"], s["q_start"], s["ctx_len"], s["blocks"], block=s["block"], out=s["out"],
                             lse=s["lse"], max_chunk=s["new_hi"], max_ctx=s["ctx_hi"] + s["new_hi"])
            return s["out"], s["lse"]
        cb.cb_block_tree_attn(s["q"], s["k_pool"], s["v_pool"], s["table"], s["ctx_len"], s["k_tree"], s["v_tree"], s["mask"], s["n_nodes"], s["blocks"],
                              block=s["block"], out=s["out"], lse=s["lse"], max_ctx=s["ctx_hi"])
        return s["out"], s["lse"]
    if kind == "pages":
        for want in (s["want"], s["back"]):
            _plain_pages(s, want)
        return s["table"], s["held"], s["free"], s["n_free"]
    if kind == "slots":
        return _plain_slots(s)
    if kind == "summary":
        return _plain_summary(s)
    if kind == "select":
        return _plain_select(s)
    return _plain_attn(s)


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without
def _selected(case, ctx):
    nb = -(-ctx // case["block"])
    return ctx - np.maximum(nb - case["n_select"], 0) * case["block"]


def work(case):
    kind, B = case["kind"], case["batch"]
    if kind == "pages":
        old, new = _page_lengths(case)
        moved = int((-(-new // PAGE) - -(-old // PAGE)).sum()) * (2 / 3 if case["tight"] else 1)
        return {"bytes": int(2 * (12 * B + 8 * moved + 8)), "flops": 0}
    new, ctx = _lengths(case)
    if kind == "slots":
        rows = int(new.sum())
        return {"bytes": (rows + case["pad"]) * 16 + int((-(-(ctx + new) // PAGE) - ctx // PAGE).sum()) * 4 + 8 * B + 4, "flops": 0}
    hkv, d = case["hkv"], case["d"]
    if kind == "summary":
        S = case["block"]
        first = ctx // S * S
        tokens = int(np.where(new > 0, ctx + new - first, 0).sum())
        blocks = int(np.where(new > 0, -(-(ctx + new) // S) - ctx // S, 0).sum())
        # the kernel's part is the blocks' own; a pass here also gives all means back as 32-bit values
        pages = int((-(-(ctx + new) // PAGE)).sum()) + 61
        return {"bytes": tokens * hkv * d * 2 + blocks * hkv * (d + 4) + pages * hkv * (d * 5 + 4), "flops": tokens * hkv * d + pages * hkv * d}
    hq = case["hq"]
    if kind == "select":
        nb = -(-ctx // case["block"])
        rows = int(new.sum())
        return {"bytes": int(nb.sum()) * (hkv * (d + 4) + 4) + rows * hq * d * 2 + B * hkv * case["n_select"] * 4, "flops": int((nb * new).sum()) * hq * d * 2}
    keys = _selected(case, ctx)
    rows = int(new.sum())
    if kind == "attn":
        seen = int((new * keys + new * (new + 1) // 2).sum())
        return {"bytes": int((keys + new).sum()) * hkv * d * 4 + rows * hq * (d * 4 + 4), "flops": 4 * hq * d * seen}
    seen = int((new * keys + 4 * new).sum())                            # a node's ancestors are a few
    return {"bytes": int((keys + new).sum()) * hkv * d * 4 + rows * hq * d * 2 + B * case["new_hi"] * hq * (d * 2 + 4), "flops": 4 * hq * d * seen}


# ---------------------------------------------------------------------------------------------------- the definition, in 64 bits
def _exact_pages(s):
    table, held, free = (s[x].cpu().numpy().astype(np.int64) for x in ("table", "held", "free"))
    stack = [int(x) for x in free[:int(s["n_free"][0])]]
    for want in (s["want"], s["back"]):
        target = -(-want.cpu().numpy().astype(np.int64) // PAGE)
        given = [int(table[b, c]) for b in range(len(held)) for c in range(target[b], held[b])]
        stack += given[::-1]
        room, asked = len(stack), 0
        for b in range(len(held)):
            if target[b] > held[b]:
                asked += int(target[b] - held[b])
                if asked > room:
                    continue
                for c in range(held[b], target[b]):
                    table[b, c] = stack.pop()
            held[b] = target[b]
        free[:len(stack)] = stack                                      # what lies above the top stays what it was
    return _dev(table), _dev(held), _dev(free), _dev(np.array([len(stack)]))


def exact(case, seed):
    kind, s, f8 = case["kind"], prepare(case, seed), torch.float64
    if kind == "pages":
        return _exact_pages(s)
    ctx, start, bt = s["ctx_len"].tolist(), s["q_start"].tolist(), s["table"].cpu().numpy()
    if kind == "slots":
        res = {x: np.full(s["n_rows"], -1, np.int64) for x in ("slots", "positions", "seqs")}
        for b, c in enumerate(ctx):
            pos = c + np.arange(start[b + 1] - start[b])
            rows = slice(start[b], start[b + 1])
            res["slots"][rows], res["positions"][rows], res["seqs"][rows] = bt[b, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE, pos, b
        return {k: _dev(v, torch.int64 if k == "slots" else torch.int32) for k, v in res.items()}
    S = case["block"]
    if kind == "summary":
        value, scale = s["k_mean"].to(f8) * 0.0, s["k_scale"].to(f8)
        flat = s["k_pool"].view(-1, case["hkv"], case["d"])
        for b, hi in enumerate(s["to_len"].tolist()):
            if hi == ctx[b]:
                continue
            lo = ctx[b] // S * S
            t = np.arange(lo, hi)
            rows = flat[_dev(bt[b, t // PAGE].astype(np.int64) * PAGE + t % PAGE, torch.int64)].to(f8)
            full = (hi - lo) // S
            means = list(rows[:full * S].view(full, S, case["hkv"], case["d"]).mean(1).unbind(0))
            if (hi - lo) % S:
                means.append(rows[full * S:].mean(0))
            mean = torch.stack(means)
            at = _dev(bt[b, (lo // S + np.arange(len(means))) * S // PAGE], torch.int64)
            peak = mean.abs().max(-1, keepdim=True)[0]                  # (an element half way between two steps is so in 64 bits too)
            value[at], scale[at] = torch.round(127.0 * mean / peak) * (peak / 127.0), peak[..., 0] / 127.0
        return dict(k_mean=value, k_scale=scale)
    Hkv, G, K, D = case["hkv"], case["hq"] // case["hkv"], case["n_select"], case["d"]
    node_rows = s["n_nodes"].tolist() if case["tree"] else None
    queries = lambda b: s["q"][b, :node_rows[b]] if case["tree"] else s["q"][start[b]:start[b + 1]]
    if kind == "select":
        res = np.full((case["batch"], Hkv, K), -1, np.int64)
        for b, c in enumerate(ctx):
            nb = -(-c // S)
            first = _dev(bt[b, np.arange(nb) * S // PAGE], torch.int64)
            x = queries(b).to(torch.float32)
            for h in range(Hkv):
                y = x[:, h * G:h * G + G].reshape(-1, D)
                eighth = torch.round(y * (torch.full((1,), 127.0, device=DEV) / y.abs().max())).to(f8)
                best = (eighth @ s["k_mean"][first, h].to(f8).t()).max(0)[0]
                score = (best.to(torch.float32) * s["k_scale"][first, h]).cpu().numpy() if nb else np.zeros(0, np.float32)
                forced = sorted(set([0] if nb else []) | set(range(max(0, nb - 2), nb)))
                others = sorted((j for j in range(nb) if j not in forced), key=lambda j: (-score[j], j))
                chosen = sorted(forced + others[:K - len(forced)])
                res[b, h, :len(chosen)] = chosen
        return _dev(res)
    kp, vp = s["k_pool"].view(-1, Hkv, D), s["v_pool"].view(-1, Hkv, D)
    lists = s["blocks"].cpu().numpy()
    out, lse = torch.zeros(s["q"].shape, device=DEV, dtype=f8), torch.zeros(s["lse"].shape, device=DEV, dtype=f8)
    for b, c in enumerate(ctx):
        x = queries(b).to(f8)
        n = x.shape[0]
        for h in range(Hkv):
            ids = lists[b, h][lists[b, h] >= 0]
            t = np.concatenate([np.arange(j * S, min((j + 1) * S, c)) for j in ids] + ([] if case["tree"] else [np.arange(c, c + n)])).astype(np.int64)
            at = _dev(bt[b, t // PAGE].astype(np.int64) * PAGE + t % PAGE, torch.int64)
            k, v = kp[at, h].to(f8), vp[at, h].to(f8)
            old = len(t) - (0 if case["tree"] else n)
            hidden = torch.zeros(n, len(t) + (n if case["tree"] else 0), device=DEV, dtype=torch.bool)
            if case["tree"]:
                k, v = torch.cat((k, s["k_tree"][b, :n, h].to(f8))), torch.cat((v, s["v_tree"][b, :n, h].to(f8)))
                word = s["mask"][b, :n].cpu().numpy().view(np.uint32)
                hidden[:, old:] = _dev(np.unpackbits(word.view(np.uint8), axis=-1, bitorder="little")[:, :n] == 0, torch.bool)
            else:
                hidden[:, old:] = torch.ones(n, n, device=DEV, dtype=torch.bool).triu(1)
            for g in range(h * G, h * G + G):
                z = (x[:, g] @ k.t() / math.sqrt(D)).masked_fill(hidden, -math.inf)
                o, e = torch.softmax(z, 1) @ v, torch.logsumexp(z, 1)
                if case["tree"]:
                    out[b, :n, g], lse[b, g, :n] = o, e
                else:
                    out[start[b]:start[b + 1], g], lse[start[b]:start[b + 1], g] = o, e
    return out, lse
