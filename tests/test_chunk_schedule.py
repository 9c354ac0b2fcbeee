"""Chunk attention's split over the persistent CTAs and the search for a row's sequence, from the kernels' own headers compiled for the host (a
warp's 32 lanes emulated), against a plain restatement."""
import os
import subprocess

import numpy as np
import pytest

from tests.test_attn_schedule_pairs import _SHIM as _WARP

_SHIM = _WARP.split('#include "cb_attn_sched32.cuh"')[0] + r"""
inline int __clz(int x) { return x == 0 ? 32 : __builtin_clz((unsigned)x); }
#include "cb_chunk_sched.cuh"
int main() {
    int what;
    while (scanf("%d", &what) == 1) {
        if (what == 0) {                                       // sequences of rows
            int B, n;
            if (scanf("%d %d", &B, &n) != 2) return 1;
            std::vector<int> q(B + 1);
            std::vector<int> ctx(B);
            for (int& x : q) if (scanf("%d", &x) != 1) return 1;
            for (int b = 0; b < B; ++b) ctx[b] = 7 * b + 1;
            for (int r = 0; r < n; ++r) {
                int got = -2, other = -2;
                warp([&](int lane) {
                    int q0 = 0, q1 = 0, c = 0;
                    const int b = cb_find_sequence(q.data(), B, r, lane, ctx.data(), &q0, &q1, &c);
                    if (b >= 0 && (q0 != q[b] || q1 != q[b + 1] || c != ctx[b])) got = other = -3;
                    else if (lane == 0) got = b;
                    else if (lane == 31) other = b;
                });
                if (got != other) { printf("lanes differ\n"); return 1; }
                printf("%d ", got);
            }
        } else if (what == 3) {                               // few units, many CTAs each
            CbChunkParams p = {};
            if (scanf("%d %d %d %d %d %d", &p.B, &p.G, &p.Hkv, &p.D, &p.nc, &p.max_keys) != 6) return 1;
            std::vector<int> q(p.B + 1), c(p.B);
            for (int& x : q) if (scanf("%d", &x) != 1) return 1;
            for (int& x : c) if (scanf("%d", &x) != 1) return 1;
            p.q_start = q.data(); p.ctx_len = c.data(); p.n_rows = p.max_chunk = q[p.B];
            p.NPT = CB_MT / p.G; p.one = 1;
            p.cs = cb_chunk_pick_share((long long)p.B * p.Hkv, (p.max_keys + 127) / 128, p.nc);
            printf("%d ", p.cs);
            for (int k = 0; p.cs && k < p.B * p.Hkv * p.cs; ++k) {
                CbChunkUnit u;
                CbChunkShape s;
                int np = 0;
                if (cb_chunk_share(p, k / p.cs / p.Hkv, k / p.cs % p.Hkv, k % p.cs, &u, &s, &np)) printf("%d %d %d %d %d %d %d ", k, u.b, u.kh, u.t0, u.t1, s.tiles(0), np);
            }
        } else if (what == 1) {
            long long n;
            int a, b;
            if (scanf("%lld %d %d", &n, &a, &b) != 3) return 1;
            printf("%lld ", cb_floor_sum(n, a, b));
        } else {
            CbChunkParams p = {};
            const bool pairs = what == 4;
            if (scanf("%d %d %d %d %d %d %d %d", &p.B, &p.G, &p.Hkv, &p.D, &p.nc, &p.max_chunk, &p.max_keys, &p.n_rows) != 8) return 1;
            std::vector<int> q(p.B + 1), c(p.B);
            for (int& x : q) if (scanf("%d", &x) != 1) return 1;
            for (int& x : c) if (scanf("%d", &x) != 1) return 1;
            p.q_start = q.data(); p.ctx_len = c.data();
            p.NPT = CB_MT / p.G; p.one = p.max_chunk <= p.NPT;
            CbAttnParams w = {};
            w.D = p.D;
            cb_attn_weights(w);
            p.w1 = w.w1; p.w2 = w.w2; p.d1 = w.d1; p.d2 = w.d2;
            int error = 0;
            for (int k = 0; k < p.nc; ++k) {
                CbChunkWalker wk = {};
                CbChunkCuts cuts;
                warp([&](int lane) {
                    CbChunkWalker x;
                    CbChunkCuts t;
                    int err = 0;
                    cb_chunk_range(p, k, lane, &x, &t, &err);
                    if (err) error = err;
                    if (lane == 7) { wk = x; cuts = t; }
                });
                CbChunkUnit u;
                bool heads = false;
                while (pairs ? wk.next_pair(p, &u, &heads) : wk.next(p, &u)) {
                    const CbChunkShape& s = wk.s;
                    const int tiles = s.tiles(u.rg), wt = s.wt(u.rg), cf = cuts.of(u.first);
                    const int np = cuts.total >= (long long)p.nc * wt ? cuts.of(u.first + (long long)(tiles - 1) * wt) - cf + 1 : tiles;
                    printf("%d %d %d %d %d %d %d %d %d %d %d %d ", k, u.b, u.kh, u.rg, u.t0, u.t1, tiles, heads ? 3 : (s.two_rows(u.rg) ? 2 : 1), s.row0, s.end(u.rg), cf, np);
                }
            }
            printf("\n%d", error);
        }
        printf("\n");
    }
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    from paper_2511_21699_b200 import build as b
    d = tmp_path_factory.mktemp("chunk")
    (d / "shim.cpp").write_text(_SHIM)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-w", "-I", os.path.join(cuda, "include"), "-I", os.path.join(b.ROOT, "include"), "-I", b.CSRC,
                           str(d / "shim.cpp"), "-o", str(d / "shim")])

    def run(text):
        r = subprocess.run([str(d / "shim")], input=text, capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, (r.returncode, r.stdout[-200:])
        return r.stdout
    return run


@pytest.mark.parametrize("B", [1, 2, 31, 32, 33, 100, 1024, 1025, 2500])
def test_sequence_of_a_row(shim, B):
    rng = np.random.default_rng(B)
    n = np.where(rng.random(B) < 0.5, 0, rng.integers(0, 4, B))
    q = 3 + np.concatenate([[0], np.cumsum(n)])
    rows = int(q[-1]) + 4
    got = np.array(shim("0 %d %d %s\n" % (B, rows, " ".join(map(str, q)))).split(), int)
    assert np.array_equal(got, np.searchsorted(q[:-1], np.arange(rows), side="right") - 1)


def test_floor_sum(shim):
    rng = np.random.default_rng(0)
    cases = [(0, 5, 7), (1, 0, 0), (1, 256, 300), (3, 128, 127)] + [(int(rng.integers(0, 400)), int(rng.choice([16, 18, 32, 36, 42, 50, 64, 84, 128, 256])),
                                                                     int(rng.integers(0, 40000))) for _ in range(200)]
    got = [int(x) for x in shim("".join("1 %d %d %d\n" % c for c in cases)).split()]
    assert got == [sum((a * i + b) // 128 for i in range(n)) for n, a, b in cases]


def _plain(G, hkv, D, nc, max_chunk, q, ctx):
    """[(cta, b, kh, rg, t0, t1, tiles, row tiles, first row, keys seen, cta of the first tile, ctas)], tile by tile."""
    npt = 128 // G
    one = max_chunk <= npt
    tg = npt if one else 2 * npt
    w = {128: {1: (4, 3), 2: (6, 2)}, 64: {1: (1, 0), 2: (2, 0)}}[D]
    units, at = [], 0
    for b in range(len(ctx)):
        n = q[b + 1] - q[b]
        for rg in range(-(-n // tg)):
            nrt = 2 if not one and n - rg * tg > npt else 1
            wt, dec = w[nrt]
            pad = 3 * wt if nrt == 2 else 2 * wt
            end = ctx[b] + min(n, (rg + 1) * tg)
            tiles = -(-end // 128)
            for kh in range(hkv):
                units.append((b, kh, rg, nrt, q[b], end, tiles, wt, at + pad + dec))
                at += pad + tiles * wt
    bounds = [at * c // nc for c in range(nc + 1)]
    out = []
    for b, kh, rg, nrt, row0, end, tiles, wt, first in units:
        owner = np.searchsorted(bounds, first + wt * np.arange(tiles), side="right") - 1
        holders = np.unique(owner)
        for c in holders:
            mine = np.nonzero(owner == c)[0]
            out.append((int(c), b, kh, rg, int(mine[0]), int(mine[-1]) + 1, tiles, nrt, row0, end, int(owner[0]), len(holders)))
    return sorted(out)


@pytest.mark.parametrize("G,hkv,D,new,ctx", [
    (1, 32, 128, [1], [4095]), (4, 8, 128, [1] * 64, list(range(120, 8200, 128))), (4, 4, 64, [0, 509, 1, 64, 0, 200], [3, 0, 5000, 640, 9, 0]),
    (8, 8, 128, [8192], [0]), (7, 4, 128, [1000, 3, 18, 19, 36, 37], [77, 0, 5, 250, 1, 128]), (5, 1, 64, [2000, 1], [31, 9000]), (16, 3, 128, [40, 8, 9], [0, 1, 2]),
    (3, 2, 64, [0, 0, 0], [1, 2, 3]), (1, 1, 128, [1], [0]), (2, 2, 128, [300] * 3, [0, 128, 500]), (1, 40, 64, [129, 128, 127, 1], [0, 0, 0, 0]),
    (4, 1, 128, [1] * 100, [5] * 100), (6, 2, 128, [900, 0, 5000], [200, 7, 60]), (16, 1, 64, [2500, 3], [150000, 50]), (3, 4, 128, [1] * 33 + [4000] + [0] * 40 + [2], [9] * 75),
])
def test_who_works_on_what(shim, G, hkv, D, new, ctx):
    q = np.concatenate([[0], np.cumsum(new)]).tolist()
    for nc in (148, 160, 7, 1):
        for max_chunk in sorted({max(max(new), 1), max(q[-1], 1)}):
            text = "2 %d %d %d %d %d %d %d %d %s %s\n" % (len(new), G, hkv, D, nc, max_chunk, 1 << 30, q[-1], " ".join(map(str, q)), " ".join(map(str, ctx)))
            units, error = shim(text).split("\n")[:2]
            got = sorted(tuple(int(y) for y in x) for x in np.array(units.split(), np.int64).reshape(-1, 12))
            assert int(error) == 0
            want = _plain(G, hkv, D, nc, max_chunk, q, ctx)
            assert got == want
            # whole units of one row tile taken two heads at a time, from the front, wherever the next head's is whole here too
            flat = sorted(want, key=lambda x: (x[0], x[1], x[3], x[2]))
            paired, k = [], 0
            while k < len(flat):
                x = flat[k]
                y = flat[k + 1] if k + 1 < len(flat) else None
                both = (y is not None and x[7] == 1 and (x[4], x[5]) == (0, x[6]) and (y[0], y[1], y[2], y[3], y[4], y[5]) == (x[0], x[1], x[2] + 1, x[3], 0, x[6]))
                paired.append(x[:7] + (3,) + x[8:] if both else x)
                k += 1 + both
            units, _ = shim(text.replace("2 ", "4 ", 1)).split("\n")[:2]
            assert [tuple(int(y) for y in x) for x in np.array(units.split(), np.int64).reshape(-1, 12)] == paired
            have = sorted((x[1], x[2], x[3], t) for x in got for t in range(x[4], x[5]))    # every tile once
            assert len(have) == len(set(have)) == sum(x[6] for x in {(y[1], y[2], y[3]): y for y in got}.values())


def test_sequences_that_are_left_out(shim):
    from paper_2511_21699_b200 import _lib
    for q, ctx, left, code in (([0, 3, 5, 9], [1, -1, 2], 1, _lib.CB_ERR_INVALID_ARG), ([0, 3, 2, 9], [1, 1, 2], (1, 2), _lib.CB_ERR_INVALID_ARG),   # seven tokens are more than max_chunk
                              
                               ([0, 3, 5, 99], [1, 1, 2], 2, _lib.CB_ERR_INVALID_ARG), ([-2, 3, 5, 9], [1, 1, 2], 0, _lib.CB_ERR_INVALID_ARG),
                               ([0, 3, 5, 9], [1, 999, 2], 1, _lib.CB_ERR_KV_FULL), ([0, 3, 5, 9], [1, 1, 2 ** 31 - 1], 2, _lib.CB_ERR_KV_FULL),
                               ([0, 6, 7, 9], [1, 1, 2], 0, _lib.CB_ERR_INVALID_ARG)):
        text = "2 3 1 2 64 148 5 1000 9 %s %s\n" % (" ".join(map(str, q)), " ".join(map(str, ctx)))
        units, error = shim(text).split("\n")[:2]
        got = {int(x[1]) for x in np.array(units.split(), np.int64).reshape(-1, 12)}
        assert int(error) == code and got == {0, 1, 2} - set(np.atleast_1d(left).tolist())


@pytest.mark.parametrize("B,G,hkv,new,ctx", [(1, 1, 32, [1], [4095]), (1, 8, 8, [1], [32000]), (3, 4, 2, [1, 0, 7], [5, 10, 4000]), (1, 1, 1, [1], [0]), (2, 16, 1, [8, 3], [0, 127]),
                                             (9, 4, 8, [1] * 9, [100] * 9), (1, 1, 148, [1], [9000]), (5, 1, 40, [1] * 5, [1000] * 5)])
def test_few_units_shared_by_many(shim, B, G, hkv, new, ctx):
    """Every tile of every unit has one CTA, the CTAs of a unit are neighbours from the first on, and none is without tiles among them."""
    q = np.concatenate([[0], np.cumsum(new)])
    keys = max(n + c for n, c in zip(new, ctx))
    for nc in (148, 160):
        x = [int(y) for y in shim("3 %d %d %d 128 %d %d %s %s\n" % (B, G, hkv, nc, keys, " ".join(map(str, q)), " ".join(map(str, ctx)))).split()]
        cs, rows = x[0], np.array(x[1:], np.int64).reshape(-1, 7)
        assert 0 <= cs <= 32 and cs * B * hkv <= nc
        if cs == 0:
            assert B * hkv > 40                                   # many units already
            continue
        for b in range(B):
            for kh in range(hkv):
                mine = rows[(rows[:, 1] == b) & (rows[:, 2] == kh)]
                tiles = -(-(new[b] + ctx[b]) // 128) if new[b] else 0
                np_ = min(cs, tiles)
                assert mine[:, 0].tolist() == list(range((b * hkv + kh) * cs, (b * hkv + kh) * cs + np_))
                assert sum((list(range(t0, t1)) for t0, t1 in mine[:, 3:5]), []) == list(range(tiles))
                assert (mine[:, 4] > mine[:, 3]).all() and (mine[:, 5] == tiles).all() and (mine[:, 6] == np_).all()
