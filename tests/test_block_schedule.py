"""Attention over selected blocks: which tiles a persistent CTA works on, and which page a list names, from the kernels' own headers compiled for the host (a warp's 32
lanes emulated), against a plain restatement."""
import os
import subprocess

import numpy as np
import pytest

from tests.test_attn_schedule_pairs import _SHIM as _WARP

_SHIM = _WARP.split('#include "cb_attn_sched32.cuh"')[0] + r"""
inline int __clz(int x) { return x == 0 ? 32 : __builtin_clz((unsigned)x); }
#include "cb_chunk_sched.cuh"
#include "cb_blocks.cuh"
template <typename P> void walk(P& p, bool pairs) {
    CbAttnParams w = {};
    w.D = p.D;
    cb_attn_weights(w);
    p.w1 = w.w1; p.w2 = w.w2; p.d1 = w.d1; p.d2 = w.d2;
    p.NPT = CB_MT / p.G; p.one = p.max_chunk <= p.NPT;
    for (int k = 0; k < p.nc; ++k) {
        CbChunkWalkerT<P::kMode == 2> wk = {};
        CbChunkCuts cuts;
        warp([&](int lane) {
            CbChunkWalkerT<P::kMode == 2> x;
            CbChunkCuts t;
            int err = 0;
            cb_chunk_range(p, k, lane, &x, &t, &err);
            if (lane == 5) { wk = x; cuts = t; }
        });
        CbChunkUnit u;
        bool heads = false;
        while (pairs ? wk.next_pair(p, &u, &heads) : wk.next(p, &u)) {
            const auto& s = wk.s;
            const int tiles = s.tiles(u.rg), wt = s.wt(u.rg), cf = cuts.of(u.first);
            const int np = cuts.total >= (long long)p.nc * wt ? cuts.of(u.first + (long long)(tiles - 1) * wt) - cf + 1 : tiles;
            printf("%d %d %d %d %d %d %d %d %d %d %d %d ", k, u.b, u.kh, u.rg, u.t0, u.t1, tiles, heads ? 3 : (s.two_rows(u.rg) ? 2 : 1), s.row0, s.ctx, cf, np);
        }
    }
    printf("\n");
}
int main() {
    int what;
    while (scanf("%d", &what) == 1) {
        if (what == 0) {                                      // columns of the block table
            CbBlockLists l = {};
            int ctx, n;
            if (scanf("%d %d %d %d", &ctx, &l.n_select, &l.shift, &n) != 4) return 1;
            std::vector<int> list(l.n_select);
            for (int& x : list) if (scanf("%d", &x) != 1) return 1;
            l.blocks = list.data();
            printf("%d ", cb_seen(l, ctx));
            for (int i = 0; i < n; ++i) printf("%d ", cb_page_column(l, 0, 1, 0, cb_blocks_of(ctx, l.shift), i));
            printf("\n");
        } else {
            CbListTreeParams p = {};
            int pairs;
            if (scanf("%d %d %d %d %d %d %d %d %d", &pairs, &p.B, &p.G, &p.Hkv, &p.D, &p.nc, &p.T, &p.l.n_select, &p.l.shift) != 9) return 1;
            std::vector<int> n(p.B), c(p.B);
            for (int& x : n) if (scanf("%d", &x) != 1) return 1;
            for (int& x : c) if (scanf("%d", &x) != 1) return 1;
            p.n_nodes = n.data(); p.ctx_len = c.data(); p.max_chunk = p.T; p.max_keys = 1 << 30;
            walk(p, pairs != 0);
        }
    }
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    from paper_2511_21699_b200 import build as b
    d = tmp_path_factory.mktemp("blocks")
    (d / "shim.cpp").write_text(_SHIM)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-w", "-I", os.path.join(cuda, "include"), "-I", os.path.join(b.ROOT, "include"), "-I", b.CSRC,
                           str(d / "shim.cpp"), "-o", str(d / "shim")])

    def run(text):
        r = subprocess.run([str(d / "shim")], input=text, capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, (r.returncode, r.stdout[-200:])
        return r.stdout
    return run


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("K", [1, 3, 32])
def test_columns_of_a_list(shim, block, K):
    rng = np.random.default_rng(block + K)
    for ctx in (0, 1, 15, 16, 17, block, block * K - 1, block * K, block * K + 1, block * K * 3 + 5, 40000):
        nb = -(-ctx // block)
        lst = list(range(nb)) + [-1] * (K - nb) if nb <= K else np.append(np.sort(rng.choice(nb - 1, K - 1, replace=False)), nb - 1).tolist()
        own = 50                                                             # tokens behind the context
        pos = np.concatenate([np.arange(j * block, min((j + 1) * block, ctx)) for j in lst if j >= 0] + [ctx + np.arange(own)]).astype(int)
        pages = -(-len(pos) // 16)
        seen, *cols = [int(x) for x in shim("0 %d %d %d %d %s\n" % (ctx, K, block.bit_length() - 1, pages, " ".join(map(str, lst)))).split()]
        assert seen == len(pos) - own
        # the tokens fill whole pages up to the context's end, and go on in the page that it ends in
        assert [cols[i // 16] for i in range(len(pos))] == (pos // 16).tolist()
        assert all(i % 16 == t % 16 for i, t in enumerate(pos))


def test_entries_that_name_nothing(shim):
    got = [int(x) for x in shim("0 1000 4 6 20 -1 16 %d 15\n" % (2 ** 31 - 1)).split()]
    assert got[1:13] == [-1] * 12 and got[13:17] == [60, 61, 62, 63] and got[17:] == [64, 65, 66, 67]


def _plain(G, hkv, D, nc, T, K, shift, n, ctx):
    """[(cta, b, kh, rg, t0, t1, tiles, row tiles, first row, tokens seen, cta of the first tile, ctas)]."""
    npt = 128 // G
    one = T <= npt
    tg = npt if one else 2 * npt
    w = {128: {1: (4, 3), 2: (6, 2)}, 64: {1: (1, 0), 2: (2, 0)}}[D]
    units, at = [], 0
    for rg in range(-(-T // tg)):
        for b in range(len(ctx)):
            if rg * tg >= n[b]:
                continue
            nb = -(-ctx[b] // (1 << shift))
            seen = ctx[b] - max(nb - K, 0) * (1 << shift)
            tiles = -(-seen // 128) + 1
            nrt = 2 if not one and n[b] - rg * tg > npt else 1
            wt, dec = w[nrt]
            pad = 3 * wt if nrt == 2 else 2 * wt
            for kh in range(hkv):
                units.append((b, kh, rg, nrt, b * T, seen, tiles, wt, at + pad + dec))
                at += pad + tiles * wt
    bounds = [at * c // nc for c in range(nc + 1)]
    out = []
    for b, kh, rg, nrt, row0, seen, tiles, wt, first in units:
        owner = np.searchsorted(bounds, first + wt * np.arange(tiles), side="right") - 1
        for c in np.unique(owner):
            mine = np.nonzero(owner == c)[0]
            out.append((int(c), b, kh, rg, int(mine[0]), int(mine[-1]) + 1, tiles, nrt, row0, seen, int(owner[0]), len(np.unique(owner))))
    return sorted(out)


@pytest.mark.parametrize("G,hkv,D,T,K,shift,n,ctx", [
    (8, 8, 128, 64, 32, 6, [64] * 16, list(range(16000, 32000, 1000))), (4, 2, 64, 128, 3, 5, [128, 0, 1, 65, 33, 64], [0, 500, 96, 97, 20000, 128]),
    (16, 1, 128, 128, 10, 6, [128, 1, 17], [700, 20000, 640]), (1, 3, 64, 61, 4, 4, [61, 0, 7], [9, 8, 1000]), (7, 4, 128, 37, 20, 5, [37, 18, 19, 36], [1000, 640, 641, 0]),
    (8, 2, 128, 128, 5, 7, list(range(0, 129, 3)), list(range(0, 4300, 100))), (2, 1, 64, 100, 8, 6, [0, 0], [5, 6]), (4, 3, 128, 96, 2, 6, [96] * 70, [130] * 70),
])
def test_who_works_on_what(shim, G, hkv, D, T, K, shift, n, ctx):
    for nc in (148, 160, 7, 1):
        want = _plain(G, hkv, D, nc, T, K, shift, n, ctx)
        text = "%d %d %d %d %d %d %d %d %s %s\n" % (len(n), G, hkv, D, nc, T, K, shift, " ".join(map(str, n)), " ".join(map(str, ctx)))
        got = sorted(tuple(int(y) for y in x) for x in np.array(shim("1 0 " + text).split(), np.int64).reshape(-1, 12))
        assert got == want
        paired = [tuple(int(y) for y in x) for x in np.array(shim("1 1 " + text).split(), np.int64).reshape(-1, 12)]
        flat = sorted(x for p in paired for x in ([p, p[:2] + (p[2] + 1,) + p[3:]] if p[7] == 3 else [p]))
        assert [x[:7] for x in flat] == [x[:7] for x in want]
        assert all(x[7] != 3 or (x[4], x[5]) == (0, x[6]) for x in paired)
        have = sorted((x[1], x[2], x[3], t) for x in got for t in range(x[4], x[5]))        # every tile once
        assert len(have) == len(set(have)) == sum(x[6] for x in {(y[1], y[2], y[3]): y for y in got}.values())
