// cb_chunk_attn: entry point and the plain CUDA-core kernel.
//
// The CUDA-core kernel is a debugging aid (CB_FLAG_ATTN_CUDA_CORES): a warp per row and query head, 32 keys at a time, a key per lane for
// the scores and D / 32 columns per lane for the output; fp32 throughout.
#include <math.h>

#include <algorithm>

#include "cb_chunk.cuh"

namespace {

constexpr int kWarps = 4;

template <int D>
__global__ void __launch_bounds__(32 * kWarps) cb_chunk_cc_kernel(const CbChunkParams p) {
    constexpr int C = D / 32;
    const int lane = threadIdx.x & 31;
    const long long item = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const long long rows = (long long)p.n_rows * p.Hq;
    if (item >= rows) {                                       // behind the rows' warps, a sequence per lane: what is wrong with it
        const long long b = (item - rows) * 32 + lane;
        const int error = b < p.B ? cb_chunk_seq(p, (int)b).error : 0;
        if (error) atomicCAS(p.status, 0u, (uint32_t)error);
        return;
    }
    const int row = (int)(item / p.Hq), h = (int)(item % p.Hq), kh = h / p.G;
    int q0, q1, ctx;
    const int b = cb_find_sequence(p.q_start, p.B, row, lane, p.ctx_len, &q0, &q1, &ctx);
    if (b < 0) return;
    const CbChunkSeq s = cb_chunk_seq(p, b);
    if (s.n == 0 || row - s.row0 >= s.n) return;              // (with n = 0 row0 may be any number)
    const int keys = s.ctx + row - s.row0 + 1;
    const __nv_bfloat16* q = p.q + ((size_t)row * p.Hq + h) * D;
    float m = -INFINITY, l = 0.f, acc[C] = {};
    for (int k0 = 0; k0 < keys; k0 += 32) {
        const int key = k0 + lane;
        long long at = -1;                                    // first element of this lane's key; -1: none, or a page outside the pool
        if (key < keys) {
            const int page = p.block_table[(size_t)b * p.max_pages + key / p.P];
            if (page >= 0 && page < p.num_pages) at = (((long long)page * p.P + key % p.P) * p.Hkv + kh) * D;
        }
        float x = 0.f;
        if (at >= 0)
            for (int d = 0; d < D; d += 2) {
                const float2 kf = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p.k_pool + at + d));
                const float2 qf = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(q + d));
                x = fmaf(qf.x, kf.x, fmaf(qf.y, kf.y, x));
            }
        x = key < keys ? x * p.scale_log2 : -INFINITY;
        float mx = x;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(CB_FULL, mx, o));
        const float mn = fmaxf(m, mx), a = exp2f(m - mn), w = exp2f(x - mn);
        m = mn;
        l = l * a + w;
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] *= a;
        for (int k = 0; k < 32 && k0 + k < keys; ++k) {
            const long long v = __shfl_sync(CB_FULL, at, k);
            const float wk = __shfl_sync(CB_FULL, w, k);
            if (v < 0) continue;
#pragma unroll
            for (int c = 0; c < C; ++c) acc[c] = fmaf(wk, __bfloat162float(p.v_pool[v + lane + 32 * c]), acc[c]);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(CB_FULL, l, o);
#pragma unroll
    for (int c = 0; c < C; ++c) p.out[((size_t)row * p.Hq + h) * D + lane + 32 * c] = __float2bfloat16_rn(acc[c] / l);
    if (p.lse && lane == 0) p.lse[(size_t)row * p.Hq + h] = (m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace

extern "C" cb_status cb_chunk_attn(cb_ctx* ctx, const cb_chunk_attn_args* a, void* stream) {
    CB_CHECK_ARG(ctx && a);
    CB_CHECK_ARG(a->q && a->k_pool && a->v_pool && a->block_table && a->q_start && a->ctx_len && a->out && a->out != a->q);
    CB_CHECK_ARG(a->n_rows >= 0 && a->max_pages >= 1 && a->num_pages >= 1 && a->max_chunk >= 0 && a->max_ctx >= 0);
    const uintptr_t al = (uintptr_t)a->q | (uintptr_t)a->k_pool | (uintptr_t)a->v_pool | (uintptr_t)a->out;
    CB_CHECK_ARG((al & 15) == 0 && ((uintptr_t)a->lse & 3) == 0);
    CB_CHECK_ARG(a->scale >= 0.f && a->scale < INFINITY);     // (the kernels' running maximum is of scores times a positive number)
    if (a->n_rows == 0) return CB_OK;
    const cb_config& c = ctx->cfg;
    CbChunkParams p = {};
    p.q = (const __nv_bfloat16*)a->q; p.k_pool = (const __nv_bfloat16*)a->k_pool; p.v_pool = (const __nv_bfloat16*)a->v_pool;
    p.block_table = a->block_table; p.q_start = a->q_start; p.ctx_len = a->ctx_len;
    p.out = (__nv_bfloat16*)a->out; p.lse = a->lse;
    p.B = c.batch; p.Hq = c.n_q_heads; p.Hkv = c.n_kv_heads; p.G = c.n_q_heads / c.n_kv_heads; p.D = c.head_dim; p.P = c.page_size;
    p.max_pages = a->max_pages; p.num_pages = a->num_pages; p.n_rows = a->n_rows;
    p.max_chunk = a->max_chunk > 0 ? std::min(a->max_chunk, a->n_rows) : a->n_rows;
    const long long cap = std::min<long long>((long long)a->max_pages * c.page_size, 1ll << 30);
    p.max_keys = (int)(a->max_ctx > 0 ? std::min<long long>(a->max_ctx, cap) : cap);
    const float scale = a->scale > 0.f ? a->scale : 1.0f / sqrtf((float)c.head_dim);
    p.scale_log2 = scale * 1.4426950408889634f;
    p.status = ctx->d_status;
    cudaStream_t st = (cudaStream_t)stream;
    if (!(c.flags & CB_FLAG_ATTN_CUDA_CORES)) return cb_chunk_launch_tensor(ctx, p, st);
    const long long blocks = ((long long)p.n_rows * p.Hq + (p.B + 31) / 32 + kWarps - 1) / kWarps;
    if (blocks > 0x7FFFFFFFll) return CB_ERR_UNSUPPORTED;
    if (p.D == 128) cb_chunk_cc_kernel<128><<<(unsigned)blocks, 32 * kWarps, 0, st>>>(p);
    else cb_chunk_cc_kernel<64><<<(unsigned)blocks, 32 * kWarps, 0, st>>>(p);
    cb_count_launch(1);
    CB_CUDA(cudaGetLastError());
    return CB_OK;
}
