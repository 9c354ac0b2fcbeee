// Chunk attention: which key tiles of which rows a persistent CTA works on.
//
// As in tree attention (cb_attn.cuh) work is measured in key tiles of 128 keys, a unit is one (sequence, row group, kv head) with a row
// group of two 128-row tiles (one where the last group has no more, or all chunks fit one), and all units laid end to end, with padding in
// front of each for what starting it costs, are cut into equal ranges.  What differs: a row group sees the keys up to its own last token, so
// the units of one sequence grow along its chunk, and a chunk may have hundreds of row groups.  The order is (sequence, row group, kv head);
// where a sequence's row groups start is a sum of floor((a k + b) / 128) over k, which has a closed form, so that a CTA
// finds its first unit by a scan over the sequences and a search in one of them.  (A first form, with 64-bit divisions and lengths read twice, held
// the first copy of a launch up by 8 k cycles at batch 1 and 19 k for an 8 k prompt.)
#pragma once
#include "cb_attn.cuh"
#include "cb_chunk.cuh"

// sum over i < n of floor((a i + b) / 128), a in 1..256, b >= 0.  Everything a launch does waits for this, so divisions (a chain of 100 to 200
// cycles in 32 bits, several times that in 64) are for the head counts that need them:
//   a a multiple of 128: every term is floor(b / 128) + i a / 128;
//   a a smaller power of two, m = 128 / a: floor((a i + b) / 128) = floor((i + c) / m) with c = floor(b / a), a sum of runs of m equal terms;
//   otherwise Euclid's steps: whole multiples are taken out, what is left counts the lattice points under a line, which are the same with the
//   axes exchanged.
__device__ __forceinline__ long long cb_floor_sum(long long n, int a, int b) {
    if (n <= 0) return 0;
    if ((a & 127) == 0) return (a >> 7) * (n * (n - 1) / 2) + n * (b >> 7);
    if ((a & (a - 1)) == 0) {
        const int la = 31 - __clz(a), lm = 7 - la;
        auto runs = [&](long long x) { const long long q = x >> lm; return ((q * (q - 1) / 2) << lm) + q * (x & ((1 << lm) - 1)); };   // of floor(j / m), j < x
        const long long c = b >> la;
        return runs(n + c) - runs(c);
    }
    long long sum = 0;
    uint32_t m = 128, x = (uint32_t)a, y = (uint32_t)b;
    while (true) {
        sum += (n - 1) * n / 2 * (x / m) + n * (y / m);
        x %= m; y %= m;
        const unsigned long long top = (unsigned long long)x * n + y;
        if (top < m) return sum;
        n = (long long)cb_div((long long)top, m);
        y = (uint32_t)(top - (unsigned long long)n * m);
        const uint32_t t = m; m = x; x = t;
    }
}

// The ranges of the CTAs: range c starts at floor(total c / nc).  Positions below 2^32 (a call of 2^25 tiles) need one division.
struct CbChunkCuts {
    long long total;
    int nc;
    uint32_t q, r;            // total = q nc + r, in 32 bits
    bool small;
    __device__ __forceinline__ void init(long long t, int n) {
        total = t; nc = n; small = t >> 32 == 0;
        q = (uint32_t)t / (uint32_t)n; r = (uint32_t)t - q * (uint32_t)n;
    }
    __device__ __forceinline__ long long start(int c) const {
        if (!small) return total * c / nc;
        return (long long)((unsigned long long)q * (uint32_t)c) + cb_quot((long long)(r * (uint32_t)c), nc);   // r c < nc^2
    }
    // the range that holds position x < total
    __device__ __forceinline__ int of(long long x) const {
        if (!small) return cb_cta_of(total, nc, x);
        int c = min(max((int)(__fdividef((float)x, (float)total) * (float)nc), 0), nc - 1);      // off by one at most
        while (c > 0 && start(c) > x) --c;
        while (c + 1 < nc && start(c + 1) <= x) ++c;
        return c;
    }
};

struct CbChunkShape {
    int row0 = 0, n = 0, ctx = 0, error = 0;
    int mtn = 0, RG = 0, tg = 0;   // row tiles, row groups, tokens per row group
    int w1 = 0, w2 = 0, d1 = 0, d2 = 0;
    bool one = false;
    __device__ __forceinline__ int end(int rg) const { return ctx + min(n, (rg + 1) * tg); }                 // keys that row group rg sees
    __device__ __forceinline__ int tiles(int rg) const { return (end(rg) + CB_KT - 1) / CB_KT; }
    __device__ __forceinline__ bool two_rows(int rg) const { return !one && mtn - 2 * rg >= 2; }
    __device__ __forceinline__ int wt(int rg) const { return two_rows(rg) ? w2 : w1; }
    __device__ __forceinline__ int ov(int rg) const { return two_rows(rg) ? 3 * w2 : 2 * w1; }
    __device__ __forceinline__ int unit(int rg) const { return tiles(rg) * wt(rg) + ov(rg); }                // positions of one unit
    __device__ __forceinline__ int dec(int rg) const { return ov(rg) + (two_rows(rg) ? d2 : d1); }           // deciding position of its first tile
    // positions of one kv head's units of the row groups before r (r <= RG); all but the last group have two row tiles
    __device__ __forceinline__ long long before(int r) const {
        if (r <= 0) return 0;
        const int k = min(r, RG - 1);
        return w2 * (cb_floor_sum(k, tg, ctx + tg + CB_KT - 1) + 3ll * k) + (r == RG ? unit(RG - 1) : 0);
    }
    __device__ __forceinline__ long long weight(int Hkv) const { return RG > 0 ? Hkv * before(RG) : 0; }
};

__device__ __forceinline__ CbChunkShape cb_chunk_shape(const CbChunkParams& p, int b) {
    const CbChunkSeq q = cb_chunk_seq(p, b);
    CbChunkShape s;
    s.row0 = q.row0; s.n = q.n; s.ctx = q.ctx; s.error = q.error;
    s.mtn = (q.n + p.NPT - 1) / p.NPT;
    s.one = p.one != 0;
    s.tg = s.one ? p.NPT : 2 * p.NPT;
    s.RG = s.one ? s.mtn : (s.mtn + 1) / 2;
    s.w1 = p.w1; s.w2 = p.w2; s.d1 = p.d1; s.d2 = p.d2;
    return s;
}

// Walks the units of the range [g, g1).
struct CbChunkUnit { int b, kh, rg, t0, t1; long long first; };   // first: position of the unit's first tile's deciding position
struct CbChunkWalker {
    long long g, g1, pos;     // pos: where the current unit starts
    int b, rg, kh;
    CbChunkShape s;
    __device__ __forceinline__ bool next(const CbChunkParams& p, CbChunkUnit* u) {
        while (g < g1) {
            if (rg == s.RG) {                                 // on to the next sequence that has any
                rg = 0;
                do {
                    if (++b >= p.B) { g = g1; return false; }   // (the lengths have changed under us)
                    s = cb_chunk_shape(p, b);
                } while (s.RG == 0);
            }
            const int vt = s.unit(rg), wt = s.wt(rg), dec = s.dec(rg);
            const int v0 = (int)(g - pos), v1 = (int)min((long long)vt, v0 + (g1 - g));
            u->b = b; u->kh = kh; u->rg = rg; u->first = pos + dec;
            u->t0 = cb_tiles_of(max(v0 - dec, 0) + wt - 1, wt);
            u->t1 = cb_tiles_of(max(v1 - dec, 0) + wt - 1, wt);
            g += v1 - v0;
            if (g < g1) {                                     // the unit ends in this range
                pos += vt;
                if (++kh == p.Hkv) { kh = 0; ++rg; }
            }
            if (u->t1 > u->t0) return true;
        }
        return false;
    }
    // The same with two whole units of one row tile at a time, of neighbouring heads, where the range holds the second one's tiles as well: a chain
    // each, so that what lies between two units (some 7 k cycles of a unit of one tile) is paid once for both.
    __device__ __forceinline__ bool next_pair(const CbChunkParams& p, CbChunkUnit* u, bool* heads) {
        *heads = false;
        if (!next(p, u)) return false;
        const int tiles = s.tiles(u->rg);
        if (s.two_rows(u->rg) || u->t0 > 0 || u->t1 < tiles || u->kh + 1 >= p.Hkv || g >= g1) return true;
        const int vt = s.unit(u->rg);                         // (pos is at the next head's unit now)
        if (pos + s.dec(u->rg) + (long long)(tiles - 1) * s.wt(u->rg) >= g1) return true;
        g = min(pos + vt, g1);
        if (g < g1) {
            pos += vt;
            if (++kh == p.Hkv) { kh = 0; ++rg; }
        }
        *heads = true;
        return true;
    }
};

// This CTA's range and the walker at its start, by a whole warp (every lane gets both), and the cuts.  *error: what this lane found wrong with a
// sequence, or 0.
__device__ __forceinline__ void cb_chunk_range(const CbChunkParams& p, int cta, int lane, CbChunkWalker* w, CbChunkCuts* cuts, int* error) {
    auto shape = [&](int b) { return b < p.B ? cb_chunk_shape(p, b) : CbChunkShape{}; };
    CbChunkShape s = shape(lane);
    long long own = s.weight(p.Hkv), tot = own;
    int err = s.error;
    for (int b = 32 + lane; b - lane < p.B; b += 32) {
        const CbChunkShape t = shape(b);
        if (t.error) err = t.error;
        tot += t.weight(p.Hkv);
    }
    *error = err;
    if (p.B == 1) {                                           // lane 0 has all of it
        tot = __shfl_sync(CB_FULL, tot, 0);
    } else {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) tot += __shfl_xor_sync(CB_FULL, tot, o);
    }
    cuts->init(tot, p.nc);
    w->g = cuts->start(cta);
    w->g1 = cuts->start(cta + 1);
    if (w->g >= w->g1) return;
    long long run = 0;
    int base = 0, l = 0;
    while (p.B > 1) {                                         // ends at the sequence that holds g
        long long inc = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(CB_FULL, inc, o);
            if (lane >= o) inc += t;
        }
        const uint32_t hit = __ballot_sync(CB_FULL, w->g < run + inc);
        if (hit) {
            l = __ffs(hit) - 1;
            run = __shfl_sync(CB_FULL, run + inc - own, l);
            break;
        }
        run += __shfl_sync(CB_FULL, inc, 31);
        base += 32;
        if (base >= p.B) { w->g = w->g1; return; }            // (the lengths have changed under us)
        s = shape(base + lane);
        own = s.weight(p.Hkv);
    }
    w->b = base + l;
    // that lane's shape for all
    s.row0 = __shfl_sync(CB_FULL, s.row0, l); s.n = __shfl_sync(CB_FULL, s.n, l); s.ctx = __shfl_sync(CB_FULL, s.ctx, l);
    s.mtn = __shfl_sync(CB_FULL, s.mtn, l); s.RG = __shfl_sync(CB_FULL, s.RG, l);
    s.tg = p.one ? p.NPT : 2 * p.NPT; s.one = p.one != 0;
    s.w1 = p.w1; s.w2 = p.w2; s.d1 = p.d1; s.d2 = p.d2;
    w->s = s;
    // the last row group that starts no later: 32 candidates at a time
    const long long off = w->g - run;
    int lo = 0, n = s.RG;                                     // it is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const uint32_t hit = __ballot_sync(CB_FULL, lane * step < n && s.before(at) * p.Hkv <= off);
        const int k = 31 - __clz(hit);
        n = min(step, n - k * step);
        lo += k * step;
    }
    const long long at = s.before(lo) * p.Hkv;
    w->rg = lo;
    w->kh = (int)cb_quot(off - at, s.unit(lo));
    w->pos = run + at + (long long)w->kh * s.unit(lo);
}

// Launches of few units of one row tile (single tokens of a small batch) are not cut into ranges: unit u = (sequence, kv head) has CTAs
// u cs .. u cs + cs - 1, which take equal parts of its tiles.  A CTA then needs one sequence's lengths and next to no arithmetic before its
// first copy, and no CTA has more than one unit to see to.
__device__ __forceinline__ bool cb_chunk_share(const CbChunkParams& p, int b, int kh, int rank, CbChunkUnit* u, CbChunkShape* s, int* ctas) {
    u->b = b; u->kh = kh; u->rg = 0;
    *s = cb_chunk_shape(p, b);
    if (s->RG == 0) return false;
    const int tiles = s->tiles(0), n = min(p.cs, tiles);
    *ctas = n;
    if (rank >= n) return false;
    // (tiles below 2^23 and ranks below 32: the products fit 32 bits)
    u->t0 = (int)cb_quot((long long)(tiles * rank), n); u->t1 = (int)cb_quot((long long)(tiles * (rank + 1)), n);
    return true;
}
// How many CTAs share a unit: what the longest unit's share of tiles takes, bandwidth shared by all, and what putting the parts together
// adds (in tiles; some 0.2 each), against equal ranges, whose schedule and merging take some 6 tiles longer.  0: equal ranges.
inline int cb_chunk_pick_share(long long units, long long tiles, int num_ctas) {
    int best = 0;
    double least = (double)units * (double)(tiles + 2) / num_ctas + 6.0;
    for (int cs = 1; cs <= 32 && units * cs <= num_ctas; ++cs) {
        const double cost = (double)((tiles + cs - 1) / cs) + 0.2 * cs;
        if (cost < least) { least = cost; best = cs; }
    }
    return best;
}
