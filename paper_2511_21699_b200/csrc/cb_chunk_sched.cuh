// Chunk attention: which key tiles of which rows a persistent CTA works on.
//
// As in tree attention (cb_attn.cuh) work is measured in key tiles of 128 keys, a unit is one (sequence, row group, kv head) with a row
// group of two 128-row tiles (one where the last group has no more, or all chunks fit one), and all units laid end to end, with padding in
// front of each for what starting it costs, are cut into equal ranges.  What differs: a row group sees the keys up to its own last token, so
// the units of one sequence grow along its chunk, and a chunk may have hundreds of row groups.  The order is (sequence, row group, kv head);
// where a sequence's row groups start is a sum of floor((a k + b) / 128) over k, which has a closed form by Euclid's steps, so that a CTA
// finds its first unit by a scan over the sequences and a search in one of them.
#pragma once
#include "cb_attn.cuh"
#include "cb_chunk.cuh"

// sum over i < n of floor((a i + b) / 128), a, b >= 0: whole multiples are taken out, what is left counts the lattice points under a line, which
// are the same with the axes exchanged.
__device__ __forceinline__ long long cb_floor_sum(long long n, long long a, long long b) {
    long long sum = 0, m = 128;
    while (true) {
        if (a >= m) { sum += (n - 1) * n / 2 * (a / m); a %= m; }
        if (b >= m) { sum += n * (b / m); b %= m; }
        const long long y = a * n + b;
        if (y < m) return sum;
        n = y / m; b = y % m;
        const long long t = m; m = a; a = t;
    }
}

struct CbChunkShape {
    int row0, n, ctx, error;
    int mtn, RG, tg;          // row tiles, row groups, tokens per row group
    int w1, w2, d1, d2;
    bool one;
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
        return w2 * (cb_floor_sum(k, tg, (long long)ctx + tg + CB_KT - 1) + 3ll * k) + (r == RG ? unit(RG - 1) : 0);
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
};

// This CTA's range and the walker at its start, by a whole warp (every lane gets both); returns the positions of all units.  *error: what this
// lane found wrong with a sequence, or 0.
__device__ __forceinline__ long long cb_chunk_range(const CbChunkParams& p, int cta, int lane, CbChunkWalker* w, int* error) {
    long long tot = 0, mine = 0;
    int err = 0;
    CbChunkShape first = {};
    for (int base = 0; base < p.B; base += 32) {
        CbChunkShape s = {};
        if (base + lane < p.B) s = cb_chunk_shape(p, base + lane);
        if (base == 0) first = s;
        if (s.error) err = s.error;
        mine += s.weight(p.Hkv);
    }
    tot = mine;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) tot += __shfl_xor_sync(CB_FULL, tot, o);
    *error = err;
    w->g = cb_range_start(tot, p.nc, cta);
    w->g1 = cb_range_start(tot, p.nc, cta + 1);
    if (w->g >= w->g1) return tot;
    long long run = 0;
    for (int base = 0; base < p.B; base += 32) {
        CbChunkShape s = first;
        if (base > 0) {
            s = CbChunkShape{};
            if (base + lane < p.B) s = cb_chunk_shape(p, base + lane);
        }
        const long long own = s.weight(p.Hkv);
        long long inc = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(CB_FULL, inc, o);
            if (lane >= o) inc += t;
        }
        const long long pre = run + inc - own;
        const uint32_t hit = __ballot_sync(CB_FULL, own > 0 && w->g >= pre && w->g < pre + own);
        if (hit) {
            const int l = __ffs(hit) - 1;
            w->b = base + l;
            w->pos = __shfl_sync(CB_FULL, pre, l);
            break;
        }
        run += __shfl_sync(CB_FULL, inc, 31);
    }
    w->s = cb_chunk_shape(p, w->b);
    const long long off = w->g - w->pos;
    int lo = 0, hi = w->s.RG - 1;                             // the last row group that starts no later
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (w->s.before(mid) * p.Hkv <= off) lo = mid; else hi = mid - 1;
    }
    const long long at = w->s.before(lo) * p.Hkv;
    w->rg = lo;
    w->kh = (int)cb_div(off - at, w->s.unit(lo));
    w->pos += at + (long long)w->kh * w->s.unit(lo);
    return tot;
}
