// cb_block_attn, cb_block_tree_attn: attention over selected blocks of the cached context.
//
// The CUDA-core kernel is a debugging aid (CB_FLAG_ATTN_CUDA_CORES): a warp per row and query head, 32 keys at a time, a key per lane for the scores and
// D / 32 columns per lane for the output; fp32 throughout.
#include <math.h>

#include <algorithm>

#include "cb_blocks.cuh"
#include "cb_chunk.cuh"

namespace {

constexpr int kWarps = 4;

template <int D, typename P>
__global__ void __launch_bounds__(32 * kWarps) cb_block_cc_kernel(const P p) {
    constexpr int C = D / 32;
    constexpr bool TREE = P::kMode == 2;
    const int lane = threadIdx.x & 31;
    const long long item = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const long long rows = (long long)p.n_rows * p.Hq;
    if (item >= rows) {                                       // behind the rows' warps, a sequence per lane: what is wrong with it
        const long long b = (item - rows) * 32 + lane;
        int error = 0;
        if (b < p.B) {
            if constexpr (TREE) error = cb_tree_error(p, (int)b);
            else error = cb_chunk_seq(p, (int)b).error;
        }
        if (error) atomicCAS(p.status, 0u, (uint32_t)error);
        return;
    }
    const int row = (int)(item / p.Hq), h = (int)(item % p.Hq), kh = h / p.G;
    int b, ctx, i, own;                                       // own: new tokens (nodes) that the row may see
    if constexpr (TREE) {
        b = row / p.T; i = row % p.T;
        own = cb_tree_nodes(p, b);
        ctx = p.ctx_len[b];
        if (i >= own) {                                       // padding, or a sequence out of its bounds
            for (int c = 0; c < C; ++c) p.out[((size_t)row * p.Hq + h) * D + lane + 32 * c] = __float2bfloat16_rn(0.f);
            if (p.lse && lane == 0) p.lse[((size_t)b * p.Hq + h) * p.T + i] = 0.f;
            return;
        }
    } else {
        int q0, q1;
        b = cb_find_sequence(p.q_start, p.B, row, lane, p.ctx_len, &q0, &q1, &ctx);
        if (b < 0) return;
        const CbChunkSeq s = cb_chunk_seq(static_cast<const CbChunkParams&>(p), b);   // (its context as it is)
        if (s.n == 0 || row - s.row0 >= s.n) return;
        ctx = s.ctx; i = row - s.row0; own = i + 1;
    }
    const int nb = cb_blocks_of(ctx, p.l.shift), seen = cb_seen(p.l, ctx), keys = seen + own;
    const __nv_bfloat16* q = p.q + ((size_t)row * p.Hq + h) * D;
    float m = -INFINITY, l = 0.f, acc[C] = {};
    for (int k0 = 0; k0 < keys; k0 += 32) {
        const int key = k0 + lane;
        const __nv_bfloat16 *kp = nullptr, *vp = nullptr;     // this lane's key; null: none, or a page outside the pool
        bool vis = key < keys;
        const bool node = TREE && vis && key >= seen;
        if constexpr (TREE) {
            if (node) {
                const int j = key - seen;
                vis = (p.mask[((size_t)b * p.T + i) * p.W + (j >> 5)] >> (j & 31)) & 1u;
                kp = p.k_tree + (((size_t)b * p.T + j) * p.Hkv + kh) * D;
                vp = p.v_tree + (((size_t)b * p.T + j) * p.Hkv + kh) * D;
            }
        }
        if (vis && !node) {
            const int col = cb_page_column(p.l, b, p.Hkv, kh, nb, key / p.P);
            const int page = col >= 0 && col < p.max_pages ? p.block_table[(size_t)b * p.max_pages + col] : -1;
            if (page >= 0 && page < p.num_pages) {
                const size_t at = (((size_t)page * p.P + key % p.P) * p.Hkv + kh) * D;
                kp = p.k_pool + at; vp = p.v_pool + at;
            }
        }
        float s = 0.f;
        if (vis && kp)
            for (int d = 0; d < D; d += 2) {
                const float2 kf = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(kp + d));
                const float2 qf = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(q + d));
                s = fmaf(qf.x, kf.x, fmaf(qf.y, kf.y, s));
            }
        s = vis ? s * p.scale_log2 : -INFINITY;
        float mx = s;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(CB_FULL, mx, o));
        const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.f : mn, a = exp2f(m - ref), w = exp2f(s - ref);
        m = mn;
        l = l * a + w;
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] *= a;
        for (int k = 0; k < 32; ++k) {
            const long long v = __shfl_sync(CB_FULL, vis ? (long long)vp : 0ll, k);
            const float wk = __shfl_sync(CB_FULL, w, k);
            if (v == 0) continue;
#pragma unroll
            for (int c = 0; c < C; ++c) acc[c] = fmaf(wk, __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(v)[lane + 32 * c]), acc[c]);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(CB_FULL, l, o);
    const float inv = l > 0.f ? 1.f / l : 0.f;                // (a tree's row whose mask is empty, over no context)
#pragma unroll
    for (int c = 0; c < C; ++c) p.out[((size_t)row * p.Hq + h) * D + lane + 32 * c] = __float2bfloat16_rn(acc[c] * inv);
    if (p.lse && lane == 0) {
        const float e = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : 0.f;
        if constexpr (TREE) p.lse[((size_t)b * p.Hq + h) * p.T + i] = e;
        else p.lse[(size_t)row * p.Hq + h] = e;
    }
}

bool lists_ok(const int32_t* blocks, int32_t block, int32_t n_select) {
    return blocks && (block == 16 || block == 32 || block == 64 || block == 128) && n_select >= 1 && n_select <= CB_MAX_SELECT;
}

template <typename P>
cb_status launch_plain(const P& p, cudaStream_t st) {
    const long long blocks = ((long long)p.n_rows * p.Hq + (p.B + 31) / 32 + kWarps - 1) / kWarps;
    if (blocks > 0x7FFFFFFFll) return CB_ERR_UNSUPPORTED;
    if (p.D == 128) cb_block_cc_kernel<128><<<(unsigned)blocks, 32 * kWarps, 0, st>>>(p);
    else cb_block_cc_kernel<64><<<(unsigned)blocks, 32 * kWarps, 0, st>>>(p);
    cb_count_launch(1);
    CB_CUDA(cudaGetLastError());
    return CB_OK;
}

}  // namespace

extern "C" cb_status cb_block_attn(cb_ctx* ctx, const cb_chunk_attn_args* a, const int32_t* blocks, int32_t block, int32_t n_select, void* stream) {
    CB_CHECK_ARG(ctx && a && lists_ok(blocks, block, n_select));
    CbListParams p = {};
    const cb_status e = cb_chunk_params(ctx, a, &p);
    if (e != CB_OK || a->n_rows == 0) return e;
    p.l = {blocks, n_select, __builtin_ctz((unsigned)block)};
    cudaStream_t st = (cudaStream_t)stream;
    if (ctx->cfg.flags & CB_FLAG_ATTN_CUDA_CORES) return launch_plain(p, st);
    // 16 rows by heads at most are a stream for warps, more are tiles.  (Lists of 2,048 tokens, 8 kv heads of 128, the one and the other: 64 sequences of 8 rows 84 and 102 us, of 16 88 and
    // 102; eight of 8 10.4 and 18.3, of 16 13.6 and 18.6; one 6.3 and 13.4, 8.4 and 13.8.  The warps' kernel has no form for more; a trial one for 24 took 92 us against 103, and 16.2 against 19.7.)
    return (long long)p.max_chunk * p.G <= 16 ? cb_block_launch_token(ctx, p, st) : cb_block_launch_tensor(ctx, p, st);
}

extern "C" cb_status cb_block_tree_attn(cb_ctx* ctx, const cb_attn_args* a, const int32_t* blocks, int32_t block, int32_t n_select, void* stream) {
    CB_CHECK_ARG(ctx && a && lists_ok(blocks, block, n_select));
    CB_CHECK_ARG(a->q && a->k_pool && a->v_pool && a->block_table && a->ctx_len && a->k_tree && a->v_tree && a->tree_mask && a->n_nodes && a->out && a->out != a->q);
    CB_CHECK_ARG(a->max_pages >= 1 && a->num_pages >= 1 && a->max_ctx >= 0);
    const uintptr_t al = (uintptr_t)a->q | (uintptr_t)a->k_pool | (uintptr_t)a->v_pool | (uintptr_t)a->k_tree | (uintptr_t)a->v_tree | (uintptr_t)a->out;
    CB_CHECK_ARG((al & 15) == 0 && ((uintptr_t)a->lse & 3) == 0);
    CB_CHECK_ARG(a->scale >= 0.f && a->scale < INFINITY);
    const cb_config& c = ctx->cfg;
    if ((long long)c.batch * c.max_nodes > 0x7FFFFFFFll) return CB_ERR_UNSUPPORTED;
    CbListTreeParams p = {};
    p.q = (const __nv_bfloat16*)a->q; p.k_pool = (const __nv_bfloat16*)a->k_pool; p.v_pool = (const __nv_bfloat16*)a->v_pool;
    p.block_table = a->block_table; p.ctx_len = a->ctx_len; p.out = (__nv_bfloat16*)a->out; p.lse = a->lse;
    p.B = c.batch; p.Hq = c.n_q_heads; p.Hkv = c.n_kv_heads; p.G = c.n_q_heads / c.n_kv_heads; p.D = c.head_dim; p.P = c.page_size;
    p.max_pages = a->max_pages; p.num_pages = a->num_pages; p.n_rows = c.batch * c.max_nodes; p.max_chunk = c.max_nodes;
    const long long cap = std::min<long long>((long long)a->max_pages * c.page_size, 1ll << 30);
    p.max_keys = (int)(a->max_ctx > 0 ? std::min<long long>(a->max_ctx, cap) : cap);
    p.scale_log2 = (a->scale > 0.f ? a->scale : 1.0f / sqrtf((float)c.head_dim)) * 1.4426950408889634f;
    p.status = ctx->d_status;
    p.k_tree = (const __nv_bfloat16*)a->k_tree; p.v_tree = (const __nv_bfloat16*)a->v_tree; p.mask = a->tree_mask; p.n_nodes = a->n_nodes;
    p.T = c.max_nodes; p.W = (c.max_nodes + 31) / 32;
    p.l = {blocks, n_select, __builtin_ctz((unsigned)block)};
    cudaStream_t st = (cudaStream_t)stream;
    return c.flags & CB_FLAG_ATTN_CUDA_CORES ? launch_plain(p, st) : cb_block_launch_tensor(ctx, p, st);
}
