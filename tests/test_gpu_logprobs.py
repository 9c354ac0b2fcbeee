"""cb_logprobs and cb_accept_logprobs against the formulas in 64 bits; the alternatives' ids exactly."""
import math

import numpy as np
import pytest
import torch

from tests.operator_refs import F8, context, cuda, likelihoods

pytestmark = pytest.mark.gpu


def _check(got, x, tok, top, what=""):
    ref, bound = likelihoods(x, tok, top)
    for k, want in ref.items():
        if k == "top_ids":
            assert torch.equal(got[k].long(), want), (what, k)
        else:
            off = (got[k].to(F8) - want).abs()
            fine = (off <= bound[k]) | (got[k].to(F8) == want)    # -inf
            assert bool(fine.all()), (what, k, float((off - bound[k]).nan_to_num(0).max()))


def _logits(n, V, dtype, seed, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, V, generator=g, device="cuda") * (0.3 + spread * torch.rand(n, 1, generator=g, device="cuda"))
    return x.to(dtype), torch.randint(V, (n,), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,top", [(1, 32000, 5), (3, 1, 1), (7, 5, 5), (5, 31, 20), (4, 257, 32), (33, 5003, 0), (9, 50257, 20), (2, 128256, 32), (300, 4099, 3),
                                     (1, 151936, 0), (1000, 2048, 1), (37, 8191, 12), (40, 128256, 32), (70, 50257, 6), (150, 130001, 0), (149, 128256, 20),
                                     (18, 100003, 31)])
def test_rows(n, V, top, dtype):
    cb = context(vocab=V)
    x, tok = _logits(n, V, dtype, n + V)
    _check(cb.cb_logprobs(x, tok, top_k=top), x, tok, top)
    assert cb.cb_poll_status()[0] == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_at_odd_places(dtype):
    """A view whose rows start at every offset within 16 bytes, read through a list of rows that names some twice; rows of one CTA and of several."""
    for V, n in ((5003, 19), (60001, 11)):
        _odd_places(V, n, dtype)


def _odd_places(V, n, dtype):
    cb = context(vocab=V)
    store, _ = _logits(n, V + 6, dtype, 5)
    x = store[:, 1:V + 1]
    rows = cuda(np.random.default_rng(0).integers(0, n, 40))
    tok = cuda(np.random.default_rng(1).integers(0, V, 40))
    _check(cb.cb_logprobs(x, tok, rows=rows, top_k=7), x[rows.long()], tok, 7)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_order_of_the_alternatives(dtype):
    """Ties go to the lowest id, wherever the large elements lie: constant rows, sorted ones, all of them in one thread's elements, -0 and 0.
    The longer rows are a cluster's: ties across its CTAs too."""
    for V in (20000, 80000):
        _order(V, dtype)


def _order(V, dtype):
    cb = context(vocab=V)
    ramp = torch.arange(V, device="cuda", dtype=torch.float32)
    one = torch.zeros(V, device="cuda")
    E = 8 if dtype == torch.bfloat16 else 4
    for k in range(V // (256 * E)):                               # what thread 3 sees, and nobody else
        one[(k * 256 + 3) * E:(k * 256 + 4) * E] = 5 + 0.25 * (k % 4)
    few = torch.zeros(V, device="cuda")
    for t in range(40):                                           # what 40 threads see: more than the list holds
        for k in range(V // (256 * E)):
            few[(k * 256 + t) * E:(k * 256 + t + 1) * E] = 1 + (t + k) % 3
    zeros = torch.where(ramp % 2 == 0, -0.0, 0.0)
    x = torch.stack([torch.ones_like(ramp), ramp / 1000, -ramp / 1000, one, few, zeros, (ramp * 7919 % 11), torch.where(ramp == V - 1, 9.0, 0.0)]).to(dtype)
    tok = cuda(np.arange(8))
    for top in (1, 2, 20, 32):
        _check(cb.cb_logprobs(x, tok, top_k=top), x, tok, top, top)


def test_more_large_elements_than_the_list_holds():
    """31 threads hold some 500 large elements each and the 32nd largest of the threads' maxima is a small one."""
    V = 128256
    cb = context(vocab=V)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(2, V, generator=g, device="cuda")
    piece = torch.arange(V, device="cuda") // 4 % 256
    x[:, piece < 31] += 40
    tok = cuda([5, 6])
    _check(cb.cb_logprobs(x, tok, top_k=32), x, tok, 32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_forbidden_tokens_and_rows_without_a_value(dtype):
    V = 3001
    cb = context(vocab=V)
    x, tok = _logits(6, V, dtype, 9)
    x[0, 5:] = -math.inf                                          # five tokens left
    x[1, :] = -math.inf
    x[1, 2900] = -3.0                                             # one left: probability 1, entropy 0
    x[2, ::2] = -math.inf
    x[3] = torch.finfo(dtype).min                                 # a mask of the type's lowest value everywhere: equally likely
    x[4, :-1] = torch.finfo(dtype).min
    tok = cuda([7, 2900, 4, 9, V - 1, 0])                         # forbidden, sure, forbidden, ...
    top = 8
    got = cb.cb_logprobs(x, tok, top_k=top)
    ref, _ = likelihoods(x, tok, top)
    assert got["logprobs"][0] == -math.inf and got["logprobs"][1] == 0 and got["entropy"][1] == 0 and got["logprobs"][2] == -math.inf
    assert (got["top_logprobs"][0, 5:] == -math.inf).all()
    for k in ("logprobs", "entropy", "top_logprobs"):
        a, b = got[k].to(F8), ref[k]
        same = (a == b) | ((a - b).abs() <= 1e-5)                 # 3,001 elements: under (3001 / 256 + 40) 2^-24 + 8 * 2^-22 of the sum, 5e-6
        assert bool(same.all()), k
    assert torch.equal(got["top_ids"].long(), ref["top_ids"])
    bad = torch.full((4, V), -math.inf, device="cuda", dtype=dtype)
    bad[1, 17] = math.nan
    bad[2] = 1.0
    bad[2, 40] = math.inf
    bad[3] = 0.0
    bad[3, 0] = math.nan
    got = cb.cb_logprobs(bad, cuda([1, 1, 1, 1]), top_k=3)
    assert got["logprobs"].isnan().all() and got["entropy"].isnan().all()
    assert bool(((got["top_ids"] >= -1) & (got["top_ids"] < V)).all()) and cb.cb_poll_status()[0] == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_fewer_tokens_than_alternatives(dtype):
    for V in (1, 7, 19):
        cb = context(vocab=V)
        x, tok = _logits(4, V, dtype, V)
        got = cb.cb_logprobs(x, tok, top_k=20)
        assert (got["top_ids"][:, V:] == -1).all() and (got["top_logprobs"][:, V:] == -math.inf).all()
        _check({k: v[:, :V] if k.startswith("top") else v for k, v in got.items()}, x, tok, V, V)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,pad", [(5000, 0), (32003, 3), (100001, 1), (700001, 0)])
def test_more_equals_than_places(V, pad, dtype):
    """Rows in which thousands are as large as the K-th: constant but for a few, a handful of allowed tokens (fewer than K, in every part of the row),
    steps of equal values, and rows whose views start at odd places."""
    cb = context(vocab=V)
    x = torch.zeros(7, V + pad, device="cuda")[:, pad:]
    g = torch.Generator(device="cuda").manual_seed(V)
    at = torch.randperm(V, generator=g, device="cuda")
    x[0, at[:3]] = 2.0
    x[1] = -math.inf
    x[1, at[:11]] = torch.randn(11, generator=g, device="cuda")
    x[2] = -math.inf
    x[2, torch.tensor([0, V - 1, V // 2], device="cuda")] = 1.0    # the outermost ids
    x[3] = torch.arange(V, device="cuda") // (V // 3)
    x[4, :] = -1.0
    x[4, V - 2:] = 0.0
    x[5] = -torch.ones(V, device="cuda")
    x[5, at[:500]] = 3.0
    x[6] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.5, -math.inf)
    x = x.to(dtype)
    tok = cuda([int(at[0])] * 2 + [0, 5, 7, int(at[1]), 2])
    for top in (1, 12, 20, 32):
        _check(cb.cb_logprobs(x, tok, top_k=top), x, tok, top, top)


def test_far_apart_and_large_logits():
    V = 4096
    cb = context(vocab=V)
    x, tok = _logits(5, V, torch.float32, 2)
    x[0] *= 1e3
    x[1] += 1e4
    x[2] = x[2] * 1e-6
    x[3, 77] = 90.0
    x[4] = -1e30
    x[4, 3] = 1e30
    _check(cb.cb_logprobs(x[:4].contiguous(), tok[:4], top_k=4), x[:4], tok[:4], 4)
    got = cb.cb_logprobs(x[4:], cuda([3]), top_k=2)
    assert got["logprobs"].item() == 0 and got["entropy"].item() == 0 and got["top_ids"].tolist() == [[3, 0]]


def test_padding_bad_tokens_and_no_tokens():
    from paper_2511_21699_b200 import _lib
    V = 1000
    cb = context(vocab=V)
    x, _ = _logits(6, V, torch.float32, 3)
    tok, rows = cuda([3, -1, 5, 6, 7, -9]), cuda([5, 0, -1, 3, 0, -2])
    got = cb.cb_logprobs(x, tok, rows=rows, top_k=2)
    assert cb.cb_poll_status()[0] == 0
    live = [0, 3, 4]
    _check({k: v[live] for k, v in got.items()}, x[rows[live].long()], tok[live], 2)
    for i in (1, 2, 5):
        assert got["logprobs"][i] == 0 and got["entropy"][i] == 0 and (got["top_ids"][i] == -1).all() and (got["top_logprobs"][i] == 0).all()
    for t, r in (([3, V], None), ([0, 0], [0, 6])):
        got = cb.cb_logprobs(x, cuda(t), rows=None if r is None else cuda(r), top_k=2)
        assert cb.cb_poll_status()[0] == _lib.CB_ERR_INVALID_ARG
        assert got["logprobs"][1] == 0 and (got["top_ids"][1] == -1).all() and got["logprobs"][0] != 0
    res = dict(logprobs=torch.full((6,), 7.0, device="cuda"), entropy=torch.empty(6, device="cuda"))
    got = cb.cb_logprobs(x, None, res=res)
    assert (got["logprobs"] == 7).all()
    _check(dict(entropy=got["entropy"]), x, None, 0)
    none = cb.cb_logprobs(x, cuda(np.zeros(0)), top_k=3)
    assert none["top_ids"].shape == (0, 3) and cb.cb_poll_status()[0] == 0


@pytest.mark.parametrize("dtype,top,stride_pad", [(torch.float32, 5, 0), (torch.bfloat16, 0, 0), (torch.bfloat16, 20, 3)])
def test_after_acceptance(dtype, top, stride_pad):
    """The tokens that cb_accept emitted, from trees with verified paths."""
    import workloads as W
    from tests.harness import synthetic_trees
    cfg = W.CbConfig("lp", 6, 2, 3, 64, 2, 33, 7, 0, 1, 1, 64, (16, 16), 5001, 1.1, 0.3, (4, 8), 64)
    B, T, V = cfg.batch, cfg.max_nodes, cfg.vocab
    par, dep, _, n = synthetic_trees(cfg, full=False)
    g = torch.Generator(device="cuda").manual_seed(4)
    store = (torch.randn(B, T, V + stride_pad, generator=g, device="cuda") * 2).to(dtype)
    logits = store[:, :, :V]
    best = logits.float().argmax(-1).cpu().numpy()
    tok = np.full((B, T), -1)
    for b in range(B):
        for i in range(n[b]):                                     # three nodes in four continue their parent
            tok[b, i] = best[b, par[b, i]] if i and (i + b) % 4 else (i * 31 + b) % V
    from paper_2511_21699_b200 import Cacheback
    cb = Cacheback.from_config(cfg)
    tree = dict(tokens=cuda(tok), parent=cuda(par), depth=cuda(dep), n_nodes=cuda(n))
    acc = cb.cb_accept(tree, logits=logits)
    got = cb.cb_accept_logprobs(logits, acc, top_k=top)
    assert cb.cb_poll_status()[0] == 0
    m, nodes, toks = (acc[k].cpu().numpy() for k in ("n_accept", "accept_nodes", "out_tokens"))
    assert m.max() >= 2 and m.min() < m.max()
    for b in range(B):
        e = m[b] + 1
        at = np.concatenate([[0], nodes[b, :m[b]]])
        _check({k: v[b, :e] for k, v in got.items()}, logits[b, cuda(at, torch.int64)], acc["out_tokens"][b, :e], top, b)
        assert (got["logprobs"][b, e:] == 0).all() and (got["entropy"][b, e:] == 0).all()
        if top:
            assert (got["top_ids"][b, e:] == -1).all() and (got["top_ids"][b, :e, 0] == acc["out_tokens"][b, :e]).all()


def test_repeated_captured_and_on_another_stream():
    V, n, top = 32000, 12, 6
    cb = context(vocab=V)
    x, tok = _logits(n, V, torch.bfloat16, 8)
    want = cb.cb_logprobs(x, tok, top_k=top)
    res = {k: torch.empty_like(v) for k, v in want.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cb.cb_logprobs(x, tok, top_k=top, res=res, stream=side)
    side.synchronize()
    for k in want:
        assert torch.equal(res[k], want[k]), k
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cb.cb_logprobs(x, tok, top_k=top, res=res)
    y, t2 = _logits(n, V, torch.bfloat16, 9)
    x.copy_(y)
    tok.copy_(t2)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    _check(res, x, tok, top)


def test_refused():
    from paper_2511_21699_b200 import CachebackError
    V = 100
    cb = context(vocab=V)
    x, tok = _logits(4, V, torch.float32, 1)
    for args, kw, text in (((x.half(), tok), {}, "float32 or bfloat16"), ((x[:, :50], tok), {}, r"\[rows, vocab\]"), ((x.t(), tok), {}, r"\[rows, vocab\]"),
                           ((x, tok.long()), {}, "dtype torch.int32"), ((x, tok.repeat(2)), {}, "at most one per row"), ((x, tok), dict(top_k=33), "top_k"),
                           ((x, tok), dict(top_k=-1), "top_k"), ((x, tok), dict(rows=tok[:2]), "tokens must be"), ((x.cpu(), tok), {}, "device"),
                           ((x, tok), dict(top_k=2, res=dict(logprobs=torch.empty(4, device="cuda"), entropy=torch.empty(4, device="cuda"),
                                                             top_ids=torch.empty(4, 3, device="cuda", dtype=torch.int32),
                                                             top_logprobs=torch.empty(4, 2, device="cuda"))), "top_ids must be"),
                           ((x[:0], tok), dict(rows=tok), "at least one row"), ((x[:1].expand(4, V), tok), {}, "invalid argument")):
        with pytest.raises(CachebackError, match=text):
            cb.cb_logprobs(*args, **kw)
    with pytest.raises(CachebackError, match="batch, max_nodes, vocab"):
        cb.cb_accept_logprobs(x.view(1, 4, V), dict(accept_nodes=tok.view(1, 4), out_tokens=tok.view(1, 4)))
