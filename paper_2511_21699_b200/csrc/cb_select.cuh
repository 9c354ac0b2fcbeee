// Selection of blocks: what its two kernels share.
#pragma once
#include "cb_blocks.cuh"

struct CbSelectParams {
    const __nv_bfloat16* q;
    const int32_t *q_start, *n_nodes;
    const int8_t* mean;
    const float* scale;
    const int32_t *table, *ctx_len;
    int32_t* out;
    int B, T, Hq, Hkv, G, P, max_pages, num_pages, n_rows, max_chunk, max_ctx;
    int shift, K, n_first, n_last;
    uint32_t g_inv;           // x / G = __umulhi(x, g_inv) for the queries x of chunks up to max_chunk; 0: G is 1
    int key_words;            // words of shared memory for the keys of all blocks, a multiple of 4
    uint32_t* status;
};
// Launches the kernel for many queries; ctas: CTAs of a cluster, which share a unit's blocks.
cb_status cb_select_launch_many(const cb_ctx* ctx, const CbSelectParams& p, int ctas, cudaStream_t st);

// One (sequence, kv head).  nb: blocks to choose from; 0 where there is nothing to choose, the list being written then.
struct CbSelectUnit { int b, kh, row0, n, nb; };
__device__ __forceinline__ CbSelectUnit cb_select_unit(const CbSelectParams& p, int unit, bool first, int tid, int threads) {
    CbSelectUnit u;
    u.b = unit / p.Hkv; u.kh = unit - u.b * p.Hkv;
    int error = 0;
    if (p.q_start) {
        u.row0 = p.q_start[u.b];
        const int end = p.q_start[u.b + 1];
        u.n = end - u.row0;
        if (u.n != 0 && (u.row0 < 0 || end < u.row0 || end > p.n_rows || u.n > p.max_chunk)) error = CB_ERR_INVALID_ARG;
    } else {
        u.row0 = u.b * p.T;
        u.n = p.n_nodes[u.b];
        if (u.n < 0 || u.n > p.T) error = CB_ERR_INVALID_ARG;
    }
    const int ctx = p.ctx_len[u.b];
    if (!error && u.n != 0) error = ctx < 0 ? CB_ERR_INVALID_ARG : (ctx > p.max_ctx ? CB_ERR_KV_FULL : 0);
    u.nb = error || u.n == 0 ? 0 : cb_blocks_of(ctx, p.shift);
    if (u.nb <= p.K) {                                        // all there are
        if (first) {
            for (int k = tid; k < p.K; k += threads) p.out[(size_t)unit * p.K + k] = k < u.nb ? k : -1;
            if (error && tid == 0 && u.kh == 0) atomicCAS(p.status, 0u, (uint32_t)error);
        }
        u.nb = 0;
    }
    return u;
}
// The unit's i-th query: row i / G, head i % G of the group.
template <int D>
__device__ __forceinline__ const __nv_bfloat16* cb_select_query(const CbSelectParams& p, const CbSelectUnit& u, int i) {
    const int row = p.g_inv ? (int)__umulhi((uint32_t)i, p.g_inv) : i;
    return p.q + ((size_t)(u.row0 + row) * p.Hq + u.kh * p.G + (i - row * p.G)) * D;
}
// Largest magnitudes of eight bf16, as bits, against what there is of two.
__device__ __forceinline__ uint32_t cb_max_bits(uint32_t top, const uint4& v) {
    return __vmaxu2(top, __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)));
}
__device__ __forceinline__ float cb_whole_factor(uint32_t top_bits) { return __fdiv_rn(127.f, fmaxf(__uint_as_float(top_bits << 16), 1e-30f)); }
// Eight bf16 times r, rounded to whole numbers, as eight bytes.  Adding 1.5 * 2^23 rounds to a whole number and leaves it in the low bits (a conversion has
// a quarter of that rate).  Two roundings, as the definition has them: packed mul.rn.f32x2 and add.rn.f32x2 come out as one fused operation with one.
__device__ __forceinline__ uint2 cb_whole8(const uint4& v, float r) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t lo = __float_as_uint(__fadd_rn(__fmul_rn(__uint_as_float(w[e] << 16), r), 12582912.f));
        const uint32_t hi = __float_as_uint(__fadd_rn(__fmul_rn(__uint_as_float(w[e] & 0xFFFF0000u), r), 12582912.f));
        o[e] = __byte_perm(lo, hi, 0x0040);
    }
    return make_uint2(__byte_perm(o[0], o[1], 0x5410), __byte_perm(o[2], o[3], 0x5410));
}
// The order of scores as that of unsigned numbers.
__device__ __forceinline__ uint32_t cb_score_key(int dot, float scale) {
    float s = __int2float_rn(dot) * scale;
    if (s != s) return 0xFFFFFFFFu;                           // not a number: before all others
    if (s == 0.f) s = 0.f;                                    // -0 is 0
    const uint32_t u = __float_as_uint(s);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// The list of a unit of up to 2 THREADS blocks from its keys, by a block of THREADS, two keys a thread.  The range between the least and the largest score is cut
// into 256 equal steps, whose keys are counted; those above the step of the want-th largest are chosen, and of its own few keys, which are listed, every one finds its rank by
// looking at all others.  False: that step has more keys than the list (equal scores), or there are scores
// without bounds; nothing is written then.  scratch: 256 + 2 * kStepKeys + 2 * THREADS / 32 + 2 words, the
// first 256 and the last two zero, a barrier behind that.  Four barriers; found bit by bit, by counting barriers or by one warp alone, it took 3 to 9 k cycles instead
// of 1.5 k.
constexpr int kStepKeys = 64;
template <int THREADS>
__device__ __forceinline__ bool cb_pick_small(const CbSelectParams& p, int nb, const uint32_t* key, uint32_t* scratch, int32_t* out) {
    constexpr int WARPS = THREADS / 32;
    uint32_t *const hist = scratch, *const list = scratch + 256, *const sums = list + 2 * kStepKeys, *const listed = sums + 2 * WARPS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lo = p.n_first, hi = nb - p.n_last;
    const uint32_t left = (uint32_t)(p.K - p.n_first - p.n_last);
    const int j0 = tid, j1 = tid + THREADS;
    const bool c0 = j0 >= lo && j0 < hi, c1 = j1 >= lo && j1 < hi;
    const uint32_t k0 = c0 ? key[j0] : 0u, k1 = c1 ? key[j1] : 0u;
    uint32_t least = __reduce_min_sync(CB_FULL, min(c0 ? k0 : 0xFFFFFFFFu, c1 ? k1 : 0xFFFFFFFFu)), most = __reduce_max_sync(CB_FULL, max(k0, k1));
    if (lane == 0) { sums[warp] = least; sums[WARPS + warp] = most; }
    __syncthreads();
    {
        const uint32_t x = lane < WARPS ? sums[lane] : 0xFFFFFFFFu, y = lane < WARPS ? sums[WARPS + lane] : 0u;
        least = __reduce_min_sync(CB_FULL, x); most = __reduce_max_sync(CB_FULL, y);
    }
    // (Subtraction, multiplication and truncation keep the order; scores that are infinite or no numbers, or that far apart, are for the other way.)
    auto score = [](uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu)); };
    const float bottom = score(least), range = score(most) - bottom, factor = 255.f / range;
    if (!(range < INFINITY)) return false;
    auto step_of = [&](uint32_t k) { return (uint32_t)min((int)((score(k) - bottom) * factor), 255); };
    const uint32_t d0 = c0 ? step_of(k0) : 0u, d1 = c1 ? step_of(k1) : 0u;
    if (c0) atomicAdd(&hist[d0], 1u);
    if (c1) atomicAdd(&hist[d1], 1u);
    __syncthreads();
    // The step that holds the want-th largest, by every warp for itself: lane l has the steps 8 l .. 8 l + 7.
    uint32_t step = 256, in_step = 0, rest = 0;               // keys of that step that are wanted
    if (left > 0) {
        const uint4 x = *reinterpret_cast<const uint4*>(hist + lane * 8), y = *reinterpret_cast<const uint4*>(hist + lane * 8 + 4);
        const uint32_t c[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        uint32_t above = x.x + x.y + x.z + x.w + y.x + y.y + y.z + y.w, own = above;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t z = __shfl_down_sync(CB_FULL, above, o); if (lane + o < 32) above += z; }
        above -= own;                                         // keys in the steps of the lanes behind
        const uint32_t hit = __ballot_sync(CB_FULL, above < left && left <= above + own);
        uint32_t s = 0, n = 0, w = 0;
#pragma unroll
        for (int e = 7; e >= 0; --e) {
            if (above < left && left <= above + c[e]) { s = lane * 8 + e; n = c[e]; w = left - above; }
            above += c[e];
        }
        const int l = 31 - __clz(hit);
        step = __shfl_sync(CB_FULL, s, l); in_step = __shfl_sync(CB_FULL, n, l); rest = __shfl_sync(CB_FULL, w, l);
        if (in_step > rest) {
            if (in_step > kStepKeys) return false;
            auto note = [&](uint32_t k, int j) { const uint32_t at = atomicAdd(listed, 1u); list[2 * at] = k; list[2 * at + 1] = (uint32_t)j; };
            if (c0 && d0 == step) note(k0, j0);
            if (c1 && d1 == step) note(k1, j1);
            __syncthreads();
        }
    }
    auto chosen = [&](bool cand, uint32_t k, uint32_t d, int j) {
        if (j >= nb) return false;
        if (!cand) return true;
        if (left == 0 || d < step) return false;
        if (d > step || in_step == rest) return true;
        uint32_t rank = 0;
        for (uint32_t i = 0; i < in_step; ++i) rank += list[2 * i] > k || (list[2 * i] == k && list[2 * i + 1] < (uint32_t)j);
        return rank < rest;
    };
    const uint32_t o0 = __ballot_sync(CB_FULL, chosen(c0, k0, d0, j0)), o1 = __ballot_sync(CB_FULL, chosen(c1, k1, d1, j1));
    if (lane == 0) { sums[warp] = __popc(o0); sums[WARPS + warp] = __popc(o1); }   // (all have read the bounds there: barriers lie between)
    __syncthreads();
    uint32_t b0 = 0, b1 = 0;
    {
        const uint32_t x = lane < WARPS ? sums[lane] : 0u, y = lane < WARPS ? sums[WARPS + lane] : 0u;
        b0 = __reduce_add_sync(CB_FULL, lane < warp ? x : 0u);
        b1 = __reduce_add_sync(CB_FULL, x + (lane < warp ? y : 0u));
    }
    const uint32_t under = (1u << lane) - 1u;
    if (o0 >> lane & 1u) out[b0 + __popc(o0 & under)] = j0;
    if (o1 >> lane & 1u) out[b1 + __popc(o1 & under)] = j1;
    return true;
}

// The same for any number of blocks, by a whole block of THREADS: eight bits at a time below the highest bit in which keys differ,
// by counts of the digits, and early where a digit's keys are all wanted.  scratch: 256 + 2 * THREADS / 32 + 3 words.
template <int THREADS>
__device__ __forceinline__ void cb_pick_block(const CbSelectParams& p, int nb, const uint32_t* key, uint32_t* scratch, int32_t* out) {
    constexpr int WARPS = THREADS / 32;
    uint32_t *const hist = scratch, *const wa = scratch + 256, *const wb = wa + WARPS, *const pick = wb + WARPS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lo = p.n_first, hi = nb - p.n_last;
    uint32_t left = (uint32_t)(p.K - p.n_first - p.n_last), least = 0xFFFFFFFFu, most = 0;
    const bool any = left > 0;
    for (int j = lo + tid; j < hi; j += THREADS) { const uint32_t k = key[j]; least = min(least, k); most = max(most, k); }
    least = __reduce_min_sync(CB_FULL, least); most = __reduce_max_sync(CB_FULL, most);
    if (lane == 0) { wa[warp] = least; wb[warp] = most; }
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; ++w) { least = min(least, wa[w]); most = max(most, wb[w]); }
    uint32_t prefix = 0;                                      // of key - least
    bool from = false;                                        // all keys from the prefix on; else those above it, and `left` of its equals
    if (any)
        for (int bits = max(24 - __clz(most - least), 0), above = 32; ; above = bits, bits = max(bits - 8, 0)) {
            const int width = above - bits;                   // (the first digit has what is above it zero)
            for (int j = lo + tid; j < hi; j += THREADS) {
                const uint32_t k = key[j] - least;
                if (above >= 32 || (k >> above) == (prefix >> above)) atomicAdd(&hist[(k >> bits) & (width >= 8 ? 255u : (1u << width) - 1u)], 1u);
            }
            __syncthreads();
            if (warp == 0) {
                uint32_t c[8], sum = 0;                       // lane 0 has the largest digits
#pragma unroll
                for (int e = 0; e < 8; ++e) { c[e] = hist[255 - (lane * 8 + e)]; sum += c[e]; }
                uint32_t before = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(CB_FULL, before, o); if (lane >= o) before += y; }
                before -= sum;
                if (before < left && left <= before + sum) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (before < left && left <= before + c[e]) { pick[0] = prefix | ((uint32_t)(255 - (lane * 8 + e)) << bits); pick[1] = left - before; pick[2] = c[e]; }
                        before += c[e];
                    }
                }
            }
            __syncthreads();
            prefix = pick[0]; left = pick[1];
            from = pick[2] == left;
            if (from || bits == 0) break;
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
        }
    auto over = [&](int j) { return j < lo || j >= hi || (any && (from ? key[j] - least >= prefix : key[j] - least > prefix)); };
    auto equal = [&](int j) { return j >= lo && j < hi && any && !from && key[j] - least == prefix; };
    // In order: a run of blocks per thread, where its chosen ones go by the sums before it.
    const int run = (nb + THREADS - 1) / THREADS, j0 = min(tid * run, nb), j1 = min(j0 + run, nb);
    uint32_t gt = 0, eq = 0;
    for (int j = j0; j < j1; ++j) { gt += over(j); eq += equal(j); }
    uint32_t gs = gt, es = eq;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(CB_FULL, gs, o), z = __shfl_up_sync(CB_FULL, es, o);
        if (lane >= o) { gs += y; es += z; }
    }
    __syncthreads();
    if (lane == 31) { wa[warp] = gs; wb[warp] = es; }
    __syncthreads();
    gs -= gt; es -= eq;
    for (int w = 0; w < warp; ++w) { gs += wa[w]; es += wb[w]; }
    for (int j = j0; j < j1; ++j) {
        const bool o = over(j), e = equal(j);
        if (o || (e && es < left)) out[gs + min(es, left)] = j;
        gs += o; es += e;
    }
}
// The unit's list from its keys in shared memory, by the whole block.  scratch: cb_pick_words<THREADS> words, zero; a barrier lies behind them and the keys.
template <int THREADS>
constexpr int cb_pick_words = (256 + 2 * kStepKeys + 2 * (THREADS / 32) + 3 + 3) / 4 * 4;
template <int THREADS>
__device__ __forceinline__ void cb_pick(const CbSelectParams& p, int nb, const uint32_t* key, uint32_t* scratch, int32_t* out) {
    if (nb <= 2 * THREADS) {
        if (cb_pick_small<THREADS>(p, nb, key, scratch, out)) return;
        __syncthreads();
    }
    cb_pick_block<THREADS>(p, nb, key, scratch, out);
}

__device__ __forceinline__ void cb_cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cb_cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Address of a word of shared memory in the cluster's first CTA, and a store there.
__device__ __forceinline__ uint32_t cb_cluster_first(const void* at) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(at)));
    return r;
}
__device__ __forceinline__ void cb_cluster_store(uint32_t at, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
