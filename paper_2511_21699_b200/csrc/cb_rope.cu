// Norm of queries and keys per head, rotation by position, and where the rows go: into the paged cache (cb_chunk_append) or the tree's
// tensors (cb_tree_rope).
//
// Each element is read once and written once, so HBM bounds it; the arithmetic is some ten instructions a pair.  D / 16 lanes share a
// head and a lane holds two pieces of 8 elements that are rotated with one another (i with i + R / 2) or each in itself (neighbouring
// pairs), so a rotation needs no exchange between lanes and the norm's sum two or three shuffles.  A warp takes 4 (D = 128) or 8
// (D = 64) heads of one row, or two to four times as many; which sequence the row belongs to is found while its elements are on their way.
//
// 8,192 rows of 64 + 2 x 8 heads of 128: 68 to 71 us, 4.8 to 5.0 TB/s of the 6.5 that a copy reaches; with 64% of the issue slots busy the loads that registers leave
// room for bound it.  32 single tokens: 3.2 to 3.6 us, a launch and three dependent reads.  2,048 tree rows of 32 + 2 x 8 from a cold start: 13.9 us.
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

// Two fp32 values in one 64-bit register pair, for the packed arithmetic of sm_100.
__device__ __forceinline__ uint64_t f2_pack(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void f2_unpack(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t f2_neg(uint64_t a) { return a ^ 0x8000000080000000ull; }
__device__ __forceinline__ uint64_t f2_swap(uint64_t a) { return a >> 32 | a << 32; }

// Eight elements as four pairs of neighbours.
__device__ __forceinline__ void unpack8(const uint4& u, uint64_t* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = f2_pack(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
__device__ __forceinline__ uint4 pack8(const uint64_t* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        f2_unpack(x[i], lo, hi);
        const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
        w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// INTER: pairs are neighbours.  U: groups of heads a warp.  Seven blocks an SM (72 registers; with three groups 12 bytes are spilled, once a warp, as there is no
// loop), five of the kernels with four groups, which have the most registers: 16,384 tree rows of 64/8 heads 119 us with five, 134 with six.  With two groups 2,048 tree
// rows of 32/8 heads take 11.2 us with seven blocks, 11.8 with six, 12.0 with eight.  (The products of a row's angles and norm weights held for all its heads save a fifth
// of the arithmetic and cost 20 registers: 12 to 26% slower.)
template <int D, bool TREE, bool INTER, int U>
__global__ void __launch_bounds__(32 * kRopeWarps, U == 4 ? 5 : 7) cb_rope_kernel(const RopeParams p) {
    CB_PDL_ENTRY();
    constexpr int LPH = D / 16, HPW = 32 / LPH;               // lanes per head, heads that a warp holds side by side
    const int lane = threadIdx.x & 31, sub = lane % LPH;
    const uint32_t item = blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
    const uint32_t urow = item / (uint32_t)p.parts;
    if (urow >= (uint32_t)p.n_rows) {                         // a whole warp
        // Behind the rows' warps, a sequence per lane: a range without any row of these has no other warp to report it.
        if constexpr (!TREE) {
            const uint32_t b = (item - (uint32_t)p.n_rows * (uint32_t)p.parts) * 32u + lane;
            if (b < (uint32_t)p.B) {
                const int q0 = p.q_start[b], q1 = p.q_start[b + 1];
                if (q0 != q1 && (q0 < 0 || q1 < q0 || q1 > p.n_rows)) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
            }
        }
        return;
    }
    const int row = (int)urow, slot0 = (int)(item - urow * (uint32_t)p.parts) * (U * HPW) + lane / LPH;
    const int R = p.rope ? p.R : 0;
    const bool turned = sub < R / 16;                         // both pieces are, or neither
    int ca = 2 * sub, cb = 2 * sub + 1;
    if (turned && !INTER) { ca = sub; cb = sub + R / 16; }   // (the lanes behind these hold what lies behind R)
    // A row's heads in one count: its queries, then its keys, then its values.
    auto is_q = [&](int u) { return slot0 + u * HPW < p.Hq; };
    auto is_qk = [&](int u) { return slot0 + u * HPW < p.Hq + p.Hkv; };
    auto is_any = [&](int u) { return slot0 + u * HPW < p.Hq + 2 * p.Hkv; };
    uint4 ua[U], ub[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int slot = slot0 + u * HPW;
        const __nv_bfloat16* src = is_q(u) ? p.q + row * p.q_stride + slot * D
                                           : (is_qk(u) ? p.k + row * p.k_stride + (slot - p.Hq) * D : p.v + row * p.v_stride + (slot - p.Hq - p.Hkv) * D);
        ua[u] = ub[u] = make_uint4(0, 0, 0, 0);
        if (is_any(u)) {
            ua[u] = *reinterpret_cast<const uint4*>(src + ca * 8);
            ub[u] = *reinterpret_cast<const uint4*>(src + cb * 8);
        }
    }
    // the row's position, and its place in the cache; the same in all lanes
    long long pos = 0;
    size_t kv_row = (size_t)row;
    bool dead = false;
    if constexpr (TREE) {
        const int b = row / p.T, i = row - b * p.T;
        const int ctx = p.ctx_len[b], depth = p.depth[row];
        dead = i >= p.n_nodes[b];
        if (!dead) {
            pos = (long long)ctx + depth;
            if (pos < 0 || (p.rope && pos >= p.rope_len)) {
                dead = true;
                if (lane == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
            }
        }
    } else {
        int q0, q1, ctx;
        const int b = cb_find_sequence(p.q_start, p.B, row, lane, p.ctx_len, &q0, &q1, &ctx);
        if (b < 0) return;
        if (row < q0 || row >= q1) return;                    // behind the last sequence
        const bool bad = ctx < 0 || q0 < 0 || q1 > p.n_rows, full = (long long)ctx + q1 - q0 > (long long)p.max_pages * p.P;
        pos = (long long)ctx + row - q0;
        if (bad || full || (p.rope && pos >= p.rope_len)) {
            if (lane == 0) atomicCAS(p.status, 0u, (uint32_t)(!bad && full ? CB_ERR_KV_FULL : CB_ERR_INVALID_ARG));
            return;
        }
        const uint32_t at = (uint32_t)pos / (uint32_t)p.P;    // (a position, the sum of two lengths, is below 2^32)
        const int page = p.block_table[(size_t)b * p.max_pages + at];
        if (page < 0 || page >= p.num_pages) {
            if (lane == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
            return;
        }
        kv_row = (size_t)page * p.P + ((uint32_t)pos - at * (uint32_t)p.P);
    }
    // The angles, the same for every head of the row.  Halves: cosines and sines of this lane's eight pairs (i, i + R / 2), two pairs to a register.
    // Neighbours: a pair (x, y) and its swap (y, x) times (c, c) and (-s, s).
    uint64_t c[8], s[8];
    if (turned && !dead) {
        float fc[8], fs[8];
        const float4* rc = reinterpret_cast<const float4*>(p.rope + pos * R + 8 * sub);
        const float4* rs = reinterpret_cast<const float4*>(p.rope + pos * R + R / 2 + 8 * sub);
        *reinterpret_cast<float4*>(fc) = rc[0]; *reinterpret_cast<float4*>(fc + 4) = rc[1];
        *reinterpret_cast<float4*>(fs) = rs[0]; *reinterpret_cast<float4*>(fs + 4) = rs[1];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (INTER) { c[i] = f2_pack(fc[i], fc[i]); s[i] = f2_pack(-fs[i], fs[i]); }
            else if (i < 4) { c[i] = f2_pack(fc[2 * i], fc[2 * i + 1]); s[i] = f2_pack(fs[2 * i], fs[2 * i + 1]); }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int slot = slot0 + u * HPW;
        if (dead) {
            ua[u] = ub[u] = make_uint4(0, 0, 0, 0);
        } else {
            const __nv_bfloat16* w = is_q(u) ? p.q_norm : p.k_norm;
            uint64_t a[4], b[4];
            unpack8(ua[u], a);
            unpack8(ub[u], b);
            if (p.q_norm || p.k_norm) {                       // all lanes: the sum is by shuffles
                uint64_t s2 = f2_mul(a[0], a[0]);
#pragma unroll
                for (int i = 1; i < 4; ++i) s2 = f2_fma(a[i], a[i], s2);
#pragma unroll
                for (int i = 0; i < 4; ++i) s2 = f2_fma(b[i], b[i], s2);
                float ss, hi;
                f2_unpack(s2, ss, hi);
                ss += hi;
#pragma unroll
                for (int o = 1; o < LPH; o <<= 1) ss += __shfl_xor_sync(CB_FULL, ss, o);
                if (is_qk(u) && w) {
                    const float inv = rsqrtf(ss * (1.0f / D) + p.eps);
                    const uint64_t inv2 = f2_pack(inv, inv);
                    uint64_t wa[4], wb[4];
                    unpack8(*reinterpret_cast<const uint4*>(w + ca * 8), wa);
                    unpack8(*reinterpret_cast<const uint4*>(w + cb * 8), wb);
#pragma unroll
                    for (int i = 0; i < 4; ++i) { a[i] = f2_mul(a[i], f2_mul(inv2, wa[i])); b[i] = f2_mul(b[i], f2_mul(inv2, wb[i])); }
                }
            }
            if (is_qk(u)) {
                if (turned) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint64_t x = a[i], y = b[i];
                        if (INTER) {
                            a[i] = f2_fma(f2_swap(x), s[i], f2_mul(x, c[i]));
                            b[i] = f2_fma(f2_swap(y), s[4 + i], f2_mul(y, c[4 + i]));
                        } else {
                            a[i] = f2_fma(f2_neg(y), s[i], f2_mul(x, c[i]));
                            b[i] = f2_fma(x, s[i], f2_mul(y, c[i]));
                        }
                    }
                }
                if (w || turned) { ua[u] = pack8(a); ub[u] = pack8(b); }
            }
        }
        if (is_any(u)) {
            __nv_bfloat16* dst = is_q(u) ? p.q_out + (size_t)row * p.Hq * D + slot * D
                                         : (is_qk(u) ? p.k_out + kv_row * p.Hkv * D + (slot - p.Hq) * D : p.v_out + kv_row * p.Hkv * D + (slot - p.Hq - p.Hkv) * D);
            *reinterpret_cast<uint4*>(dst + ca * 8) = ua[u];
            *reinterpret_cast<uint4*>(dst + cb * 8) = ub[u];
        }
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

template <int D, bool TREE, int U>
cb_status launch_rope_of(RopeParams p, cudaStream_t st) {
    constexpr int per_warp = U * 32 / (D / 16);
    p.parts = (p.Hq + 2 * p.Hkv + per_warp - 1) / per_warp;
    const long long blocks = ((long long)p.n_rows * p.parts + (TREE ? 0 : (p.B + 31) / 32) + kRopeWarps - 1) / kRopeWarps;
    if (blocks * kRopeWarps > 0x7FFFFFFFll) return CB_ERR_UNSUPPORTED;
    auto kernel = p.interleaved ? cb_rope_kernel<D, TREE, true, U> : cb_rope_kernel<D, TREE, false, U>;
    CB_CUDA(cb_launch_pdl(kernel, dim3((unsigned)blocks), dim3(32 * kRopeWarps), 0, st, p));
    cb_count_launch(1);
    return CB_OK;
}
// Groups of heads per warp: one where warps are few, since a call then takes what one of them takes; more where there are plenty, since what
// belongs to the row (its sequence, position, page, angles) is found once for all of them and their loads are under way together.  us with 1, 2, 3, 4 by
// the number of groups:
//   chunks of 32/8 heads of 128  6,000  4.9, 4.4, 4.2, 4.9;  8,000  5.5, 4.5, 5.4, 5.1;  11,000  7.3, 6.8, 6.1, 5.9;  24,000  13.9, 11.3, 11.1, 12.0
//                                28,000  -, 13.5, 13.1, 13.4;  40,000  23.0, 18.0, 17.4, 18.0;  330,000  -, 145.7, 132.0, 140.4
//   of 28/4 heads of 64          6,000  4.6, 4.3, 5.0, 4.4;  8,000  5.3, 5.9, 5.1, 6.6;  11,000  7.0, 6.8, 7.1, 7.3;  24,000  13.9, 12.7, 11.6, 14.4
//                                28,000  -, 14.6, 12.9, 15.2;  40,000  22.6, 19.6, 17.2, 21.5
//   tree rows of 32/8 heads      8,000  5.1, 4.3, 5.8, 5.1;  24,000  13.0, 10.7, 11.8, 12.0;  64,000  34.2, 27.7, 29.0, 28.3;  330,000  -, 124.3, 125.2, 123.0
//   of 64/8 heads                100,000  -, 41.1, 43.0, 40.4;  160,000  -, 63.3, 65.2, 61.6;  330,000  -, 124.8, 129.9, 121.3
//   of 12/4 (20 to 16 places)    100,000  52.8, 44.9, 44.6, 52.2;  of 28/4 heads of 64  8,000  5.1, 5.4, 5.5, 6.7;  40,000  20.7, 18.0, 18.7, 21.3;  330,000  -, 138.6, 135.9, 158.9
// (Between 7,000 and 9,000 groups one or the other is ahead by how the warps fill the SMs' last round: two by up to 20%, one by up to 12%.)
template <int D, bool TREE>
cb_status launch_rope(const RopeParams& p, cudaStream_t st) {
    constexpr int per_warp = 32 / (D / 16);
    const int heads = p.Hq + 2 * p.Hkv;
    const long long groups = (long long)p.n_rows * ((heads + per_warp - 1) / per_warp);
    if constexpr (!TREE) {
        if (groups >= 28000) return launch_rope_of<D, TREE, 3>(p, st);
    } else if constexpr (D == 128) {
        if (groups >= 100000 && heads % (4 * per_warp) == 0) return launch_rope_of<D, TREE, 4>(p, st);
    }
    return groups >= 8000 ? launch_rope_of<D, TREE, 2>(p, st) : launch_rope_of<D, TREE, 1>(p, st);
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
    return ctx->cfg.head_dim == 128 ? launch_rope<128, false>(p, (cudaStream_t)stream) : launch_rope<64, false>(p, (cudaStream_t)stream);
}

extern "C" cb_status cb_tree_rope(cb_ctx* ctx, const cb_tree_rope_args* a, void* stream) {
    CB_CHECK_ARG(ctx && a && rows_ok(a->rows, ctx->cfg));
    CB_CHECK_ARG(a->tree_depth && a->n_nodes && a->ctx_len && a->q_out && a->k_out && a->v_out);
    CB_CHECK_ARG((((uintptr_t)a->q_out | (uintptr_t)a->k_out | (uintptr_t)a->v_out) & 15) == 0);
    RopeParams p = params_of(ctx, a->rows);
    p.depth = a->tree_depth; p.n_nodes = a->n_nodes; p.ctx_len = a->ctx_len;
    p.n_rows = ctx->cfg.batch * ctx->cfg.max_nodes;
    p.q_out = (__nv_bfloat16*)a->q_out; p.k_out = (__nv_bfloat16*)a->k_out; p.v_out = (__nv_bfloat16*)a->v_out;
    return ctx->cfg.head_dim == 128 ? launch_rope<128, true>(p, (cudaStream_t)stream) : launch_rope<64, true>(p, (cudaStream_t)stream);
}
