// Norm of queries and keys per head, rotation by position, and where the rows go: into the paged cache (cb_chunk_append) or the tree's
// tensors (cb_tree_rope).
//
// Each element is read once and written once, so HBM bounds it; the arithmetic is some ten instructions a pair.  D / 16 lanes share a
// head and a lane holds two pieces of 8 elements that are rotated with one another (i with i + R / 2) or each in itself (neighbouring
// pairs), so a rotation needs no exchange between lanes and the norm's sum two or three shuffles.  A warp takes 4 (D = 128) or 8
// (D = 64) heads of one row; which sequence the row belongs to is found while its elements are on their way.
#include "cb_chunk.cuh"

namespace {

constexpr int kRopeWarps = 4;

struct RopeParams {
    const __nv_bfloat16 *q, *k, *v, *q_norm, *k_norm;
    __nv_bfloat16 *q_out, *k_out, *v_out;         // k_out, v_out: the pools, or the tree's tensors
    long long q_stride, k_stride, v_stride;
    const float* rope;
    const int32_t *q_start, *ctx_len, *block_table, *depth, *n_nodes;
    float eps;
    int rope_len, R, interleaved, B, T, Hq, Hkv, P, max_pages, num_pages, n_rows;
    int parts;                                    // warps per row
    uint32_t* status;
};

__device__ __forceinline__ void unpack8(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ uint4 pack8(const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int D, bool TREE>
__global__ void __launch_bounds__(32 * kRopeWarps) cb_rope_kernel(const RopeParams p) {
    CB_PDL_ENTRY();
    constexpr int LPH = D / 16, HPW = 32 / LPH;
    const int lane = threadIdx.x & 31, sub = lane % LPH;
    const long long item = (long long)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
    const long long row64 = item / p.parts;
    if (row64 >= p.n_rows) return;                            // a whole warp
    const int row = (int)row64, slot = (int)(item % p.parts) * HPW + lane / LPH;
    // which head this is: the row's queries, then its keys, then its values
    const bool is_q = slot < p.Hq, is_k = !is_q && slot < p.Hq + p.Hkv, is_v = !is_q && !is_k && slot < p.Hq + 2 * p.Hkv;
    const int h = is_q ? slot : (is_k ? slot - p.Hq : slot - p.Hq - p.Hkv);
    const int R = p.rope ? p.R : 0;
    const bool turned = sub < R / 16;                         // both pieces are, or neither
    int ca = 2 * sub, cb = 2 * sub + 1;
    if (turned && !p.interleaved) { ca = sub; cb = sub + R / 16; }   // (the lanes behind these hold what lies behind R)
    uint4 ua = make_uint4(0, 0, 0, 0), ub = ua;
    const __nv_bfloat16* src = is_q ? p.q + row64 * p.q_stride : (is_k ? p.k + row64 * p.k_stride : p.v + row64 * p.v_stride);
    if (is_q || is_k || is_v) {
        ua = *reinterpret_cast<const uint4*>(src + (size_t)h * D + ca * 8);
        ub = *reinterpret_cast<const uint4*>(src + (size_t)h * D + cb * 8);
    }
    // the row's position, and its place in the cache; the same in all lanes
    long long pos = 0;
    size_t kv_row = row64;
    bool dead = false;
    if constexpr (TREE) {
        const int b = row / p.T, i = row % p.T;
        dead = i >= p.n_nodes[b];
        if (!dead) {
            pos = (long long)p.ctx_len[b] + p.depth[row];
            if (pos < 0 || (p.rope && pos >= p.rope_len)) {
                dead = true;
                if (lane == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
            }
        }
    } else {
        const int b = cb_find_sequence(p.q_start, p.B, row, lane);
        if (b < 0) return;
        const int q0 = p.q_start[b], q1 = p.q_start[b + 1], ctx = p.ctx_len[b];
        if (row < q0 || row >= q1) return;                    // behind the last sequence
        const bool full = (long long)ctx + q1 - q0 > (long long)p.max_pages * p.P;
        pos = (long long)ctx + row - q0;
        if (ctx < 0 || full || (p.rope && pos >= p.rope_len)) {
            if (lane == 0) atomicCAS(p.status, 0u, (uint32_t)(ctx >= 0 && full ? CB_ERR_KV_FULL : CB_ERR_INVALID_ARG));
            return;
        }
        const int page = p.block_table[(size_t)b * p.max_pages + pos / p.P];
        if (page < 0 || page >= p.num_pages) {
            if (lane == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
            return;
        }
        kv_row = (size_t)page * p.P + pos % p.P;
    }
    if (dead) {
        ua = ub = make_uint4(0, 0, 0, 0);
    } else {
        const __nv_bfloat16* w = is_q ? p.q_norm : p.k_norm;
        float a[8], b[8];
        unpack8(ua, a);
        unpack8(ub, b);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
#pragma unroll
        for (int o = 1; o < LPH; o <<= 1) ss += __shfl_xor_sync(CB_FULL, ss, o);
        if (is_q || is_k) {
            if (w) {
                const float inv = rsqrtf(ss * (1.0f / D) + p.eps);
                float wa[8], wb[8];
                unpack8(*reinterpret_cast<const uint4*>(w + ca * 8), wa);
                unpack8(*reinterpret_cast<const uint4*>(w + cb * 8), wb);
#pragma unroll
                for (int i = 0; i < 8; ++i) { a[i] *= inv * wa[i]; b[i] *= inv * wb[i]; }
            }
            if (turned) {
                float c[8], s[8];
                const float4* rc = reinterpret_cast<const float4*>(p.rope + pos * R + 8 * sub);
                const float4* rs = reinterpret_cast<const float4*>(p.rope + pos * R + R / 2 + 8 * sub);
                *reinterpret_cast<float4*>(c) = rc[0]; *reinterpret_cast<float4*>(c + 4) = rc[1];
                *reinterpret_cast<float4*>(s) = rs[0]; *reinterpret_cast<float4*>(s + 4) = rs[1];
                if (p.interleaved) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a0 = a[2 * i], a1 = a[2 * i + 1], b0 = b[2 * i], b1 = b[2 * i + 1];
                        a[2 * i] = a0 * c[i] - a1 * s[i]; a[2 * i + 1] = a1 * c[i] + a0 * s[i];
                        b[2 * i] = b0 * c[4 + i] - b1 * s[4 + i]; b[2 * i + 1] = b1 * c[4 + i] + b0 * s[4 + i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float x = a[i], y = b[i];
                        a[i] = x * c[i] - y * s[i];
                        b[i] = y * c[i] + x * s[i];
                    }
                }
            }
            if (w || turned) { ua = pack8(a); ub = pack8(b); }
        }
    }
    if (is_q || is_k || is_v) {
        __nv_bfloat16* dst = is_q ? p.q_out + (size_t)row64 * p.Hq * D : (is_k ? p.k_out : p.v_out) + kv_row * p.Hkv * D;
        *reinterpret_cast<uint4*>(dst + (size_t)h * D + ca * 8) = ua;
        *reinterpret_cast<uint4*>(dst + (size_t)h * D + cb * 8) = ub;
    }
}

// What both calls check of their rows.
bool rows_ok(const cb_qkv_rows& r, const cb_config& c) {
    const uintptr_t al = (uintptr_t)r.q | (uintptr_t)r.k | (uintptr_t)r.v | (uintptr_t)r.q_norm | (uintptr_t)r.k_norm | (uintptr_t)r.rope;
    if (!r.q || !r.k || !r.v || (al & 15)) return false;
    if ((r.q_stride | r.k_stride | r.v_stride) & 7) return false;
    if (r.q_stride < 0 || r.k_stride < 0 || r.v_stride < 0) return false;
    if (r.rope && (r.rope_len < 1 || r.rotary_dim < 16 || r.rotary_dim % 16 || r.rotary_dim > c.head_dim)) return false;
    return !(r.q_norm || r.k_norm) || r.eps >= 0.f;
}

RopeParams params_of(cb_ctx* ctx, const cb_qkv_rows& r) {
    const cb_config& c = ctx->cfg;
    RopeParams p = {};
    p.q = (const __nv_bfloat16*)r.q; p.k = (const __nv_bfloat16*)r.k; p.v = (const __nv_bfloat16*)r.v;
    p.q_norm = (const __nv_bfloat16*)r.q_norm; p.k_norm = (const __nv_bfloat16*)r.k_norm;
    p.q_stride = r.q_stride; p.k_stride = r.k_stride; p.v_stride = r.v_stride;
    p.rope = r.rope; p.rope_len = r.rope_len; p.R = r.rotary_dim; p.interleaved = r.interleaved != 0; p.eps = r.eps;
    p.B = c.batch; p.T = c.max_nodes; p.Hq = c.n_q_heads; p.Hkv = c.n_kv_heads; p.P = c.page_size;
    p.status = ctx->d_status;
    return p;
}

template <bool TREE>
cb_status launch_rope(RopeParams p, int D, cudaStream_t st) {
    const int per_warp = 32 / (D / 16);
    p.parts = (p.Hq + 2 * p.Hkv + per_warp - 1) / per_warp;
    const long long blocks = ((long long)p.n_rows * p.parts + kRopeWarps - 1) / kRopeWarps;
    if (blocks > 0x7FFFFFFFll) return CB_ERR_UNSUPPORTED;
    auto kernel = D == 128 ? cb_rope_kernel<128, TREE> : cb_rope_kernel<64, TREE>;
    CB_CUDA(cb_launch_pdl(kernel, dim3((unsigned)blocks), dim3(32 * kRopeWarps), 0, st, p));
    cb_count_launch(1);
    return CB_OK;
}

}  // namespace

extern "C" cb_status cb_chunk_append(cb_ctx* ctx, const cb_chunk_append_args* a, void* stream) {
    CB_CHECK_ARG(ctx && a && rows_ok(a->rows, ctx->cfg));
    CB_CHECK_ARG(a->q_start && a->ctx_len && a->block_table && a->q_out && a->k_pool && a->v_pool);
    CB_CHECK_ARG(a->n_rows >= 0 && a->max_pages >= 1 && a->num_pages >= 1);
    CB_CHECK_ARG((((uintptr_t)a->q_out | (uintptr_t)a->k_pool | (uintptr_t)a->v_pool) & 15) == 0);
    if (a->n_rows == 0) return CB_OK;
    RopeParams p = params_of(ctx, a->rows);
    p.q_start = a->q_start; p.ctx_len = a->ctx_len; p.block_table = a->block_table;
    p.n_rows = a->n_rows; p.max_pages = a->max_pages; p.num_pages = a->num_pages;
    p.q_out = (__nv_bfloat16*)a->q_out; p.k_out = (__nv_bfloat16*)a->k_pool; p.v_out = (__nv_bfloat16*)a->v_pool;
    return launch_rope<false>(p, ctx->cfg.head_dim, (cudaStream_t)stream);
}

extern "C" cb_status cb_tree_rope(cb_ctx* ctx, const cb_tree_rope_args* a, void* stream) {
    CB_CHECK_ARG(ctx && a && rows_ok(a->rows, ctx->cfg));
    CB_CHECK_ARG(a->tree_depth && a->n_nodes && a->ctx_len && a->q_out && a->k_out && a->v_out);
    CB_CHECK_ARG((((uintptr_t)a->q_out | (uintptr_t)a->k_out | (uintptr_t)a->v_out) & 15) == 0);
    RopeParams p = params_of(ctx, a->rows);
    p.depth = a->tree_depth; p.n_nodes = a->n_nodes; p.ctx_len = a->ctx_len;
    p.n_rows = ctx->cfg.batch * ctx->cfg.max_nodes;
    p.q_out = (__nv_bfloat16*)a->q_out; p.k_out = (__nv_bfloat16*)a->k_out; p.v_out = (__nv_bfloat16*)a->v_out;
    return launch_rope<true>(p, ctx->cfg.head_dim, (cudaStream_t)stream);
}
