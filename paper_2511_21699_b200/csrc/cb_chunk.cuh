// Packed chunks of new tokens: sequence b's are rows q_start[b] .. q_start[b + 1) at positions from ctx_len[b] on.
#pragma once
#include "cb_common.cuh"

// The last b < B with q_start[b] <= r, by the whole warp, 32 probes at a time; -1 if there is none.  With it come its rows' bounds and its cached
// length, which the last round's lanes fetch beside their probes.
__device__ __forceinline__ int cb_find_sequence(const int32_t* q_start, int B, int r, int lane, const int32_t* ctx_len, int* q0, int* q1, int* ctx) {
    int lo = 0, n = B;                                        // it is in [lo, lo + n), or there is none
    while (n > 32) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const uint32_t hit = __ballot_sync(CB_FULL, at < lo + n && q_start[at] <= r);
        if (hit == 0u) return -1;
        const int l = 31 - __clz(hit);
        n = min(step, n - l * step);
        lo += l * step;
    }
    int start = 0, end = 0, c = 0;
    if (lane < n) { start = q_start[lo + lane]; end = q_start[lo + lane + 1]; c = ctx_len[lo + lane]; }
    const uint32_t hit = __ballot_sync(CB_FULL, lane < n && start <= r);
    if (hit == 0u) return -1;
    const int l = 31 - __clz(hit);
    *q0 = __shfl_sync(CB_FULL, start, l); *q1 = __shfl_sync(CB_FULL, end, l); *ctx = __shfl_sync(CB_FULL, c, l);
    return lo + l;
}

// What attention of packed chunks is given.
struct CbChunkParams {
    const __nv_bfloat16 *q, *k_pool, *v_pool;
    const int32_t *block_table, *q_start, *ctx_len;
    __nv_bfloat16* out;
    float* lse;
    int B, Hq, Hkv, G, D, P, max_pages, num_pages, n_rows;
    int max_chunk, max_keys;  // bounds of a sequence's new tokens and of all its tokens
    float scale_log2;         // softmax scale * log2(e)
    uint32_t* status;
    // the tensor-core kernel's split (cb_chunk_sched.cuh)
    int NPT;                  // tokens per row tile = 128 / G
    uint32_t g_inv;           // x / G = x * g_inv >> 16 for x < 256
    int one;                  // every chunk fits one row tile, by max_chunk
    int nc;                   // persistent CTAs
    int cs;                   // > 0: few units, so many CTAs share each (cb_chunk_share); 0: equal ranges of the positions
    uint32_t cs_inv, hkv_inv; // x / cs = __umulhi(x, cs_inv) for x < 2^16, and for Hkv
    int w1, w2, d1, d2;       // positions per key tile of a unit with one or two row tiles, and which of them decides whose tile it is
    float* part;              // partial outputs of units shared between CTAs; tickets and turn as in tree attention, whose scratch this is
    uint32_t *part_ticket, *part_turn;
};

// A sequence's chunk as attention sees it.  n = 0: nothing to do, or nothing that may be done (error: why).
struct CbChunkSeq { int row0, n, ctx, error; };
__device__ __forceinline__ CbChunkSeq cb_chunk_seq(const CbChunkParams& p, int b) {
    const int q0 = p.q_start[b], q1 = p.q_start[b + 1], ctx = p.ctx_len[b];
    CbChunkSeq s = {q0, 0, 0, 0};
    if (q0 == q1) return s;
    if (q0 < 0 || q1 < q0 || q1 > p.n_rows || q1 - q0 > p.max_chunk || ctx < 0) s.error = CB_ERR_INVALID_ARG;
    else if (ctx > p.max_keys - (q1 - q0)) s.error = CB_ERR_KV_FULL;
    else { s.n = q1 - q0; s.ctx = ctx; }
    return s;
}

cb_status cb_chunk_launch_tensor(cb_ctx* ctx, const CbChunkParams& p, cudaStream_t st);
