// Block summaries and the selection of blocks by them.
//
// cb_block_summary.  The mean of a block's keys, in 64 bits: a sum of up to 128 bf16 values is exact there (8-bit mantissas, unless exponents lie more than
// 2^38 apart), so a block's tokens may be dealt to warps, a block may be summarised token by token or all at once, and the bits are the same.  A CTA takes
// a block and 256 channels (two heads of 128 or four of 64): its eight warps take every eighth token, 512 contiguous bytes of it each, all of a warp's
// loads under way at once; the warps' sums are put together in shared memory, a channel per thread.  Memory bounds it: the keys are read once.
//
// cb_block_select.  A CTA per (sequence, kv head).  The queries become whole numbers of a common scale, the summaries are whole numbers already, so that
// the scores are exact and the choice is the same however the work is cut.
#include <algorithm>
#include <mutex>

#include "cb_blocks.cuh"
#include "cb_scan.cuh"

namespace {

// ------------------------------------------------------------------------------------------------ summaries
constexpr int kSumThreads = 256;

struct SummaryParams {
    const __nv_bfloat16* k_pool;
    const int32_t *table, *from, *to;
    int8_t* mean;
    float* scale;
    int B, Hkv, P, max_pages, num_pages;
    uint32_t* status;
};

template <int D, int S>
__global__ void __launch_bounds__(kSumThreads) cb_block_summary_kernel(const SummaryParams p) {
    constexpr int HG = 256 / D, LH = D / 8, T = S / 8;        // heads of a CTA, lanes of a head, tokens of a warp
    extern __shared__ int32_t s_sums[];                       // [2][B]
    __shared__ long long s_scratch[66];
    __shared__ double s_part[8][256];                         // a warp's sums: channel lane * 8 + e at e * 32 + lane
    __shared__ unsigned long long s_top[8][HG];
    __shared__ __align__(16) int8_t s_out[256];
    CB_PDL_ENTRY();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int error = 0;
    cb_block_sums<kSumThreads>(p.B, s_sums, s_sums + p.B, s_scratch, [&](int b, int* blocks, int*) {
        const int lo = p.from[b], hi = p.to[b];
        if (lo >= hi) return;
        if (lo < 0) error = CB_ERR_INVALID_ARG;
        else if (hi > (long long)p.max_pages * p.P) error = CB_ERR_KV_FULL;
        else *blocks = (hi - 1) / S - lo / S + 1;
    });
    if (error && blockIdx.x == 0) atomicCAS(p.status, 0u, (uint32_t)error);
    const int groups = (p.Hkv + HG - 1) / HG;
    const long long items = (long long)s_sums[p.B - 1] * groups;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const int at = (int)(item / groups), h0 = (int)(item % groups) * HG;
        const int b = cb_upper(s_sums, p.B, at);
        const int blk = p.from[b] / S + at - (b > 0 ? s_sums[b - 1] : 0);
        const int n = min(S, p.to[b] - blk * S);
        const int32_t* pages = p.table + (size_t)b * p.max_pages + blk * (S / 16);
        const int page = lane < (n + 15) / 16 ? pages[lane] : 0;
        const bool good = __all_sync(CB_FULL, page >= 0 && page < p.num_pages);
        const int head = h0 + lane / LH;
        double sum[8] = {};
        if (good) {
            uint4 v[T];
#pragma unroll
            for (int k = 0; k < T; ++k) {
                const int t = warp + 8 * k;
                const int pg = __shfl_sync(CB_FULL, page, t >> 4);
                v[k] = make_uint4(0, 0, 0, 0);
                if (t < n && head < p.Hkv) v[k] = *reinterpret_cast<const uint4*>(p.k_pool + (((size_t)pg * p.P + (t & 15)) * p.Hkv + head) * D + (lane % LH) * 8);
            }
#pragma unroll
            for (int k = 0; k < T; ++k) {
                const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sum[2 * e] += (double)__uint_as_float(w[e] << 16);
                    sum[2 * e + 1] += (double)__uint_as_float(w[e] & 0xFFFF0000u);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s_part[warp][e * 32 + lane] = sum[e];
        __syncthreads();
        double m = 0.0;
#pragma unroll
        for (int w = 0; w < 8; ++w) m += s_part[w][tid];
        m = __ddiv_rn(m, (double)n);
        // the largest magnitude as bits: NaN is above infinity there
        unsigned long long top = (unsigned long long)__double_as_longlong(m) & 0x7FFFFFFFFFFFFFFFull;
#pragma unroll
        for (int o = LH / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(CB_FULL, top, o));
        if (lane % LH == 0) s_top[warp][lane / LH] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) top = max(top, s_top[w][lane / LH]);
        const double a = __longlong_as_double((long long)top);
        const bool finite = top < 0x7FF0000000000000ull;
        const int q = finite ? __double2int_rn(__ddiv_rn(__dmul_rn(m, 127.0), fmax(a, 1e-30))) : 0;
        s_out[lane * 8 + warp] = (int8_t)q;
        const int first = __shfl_sync(CB_FULL, page, 0);
        if (good && warp == 0 && lane % LH == 0 && head < p.Hkv)
            p.scale[(size_t)first * p.Hkv + head] = finite ? (float)__ddiv_rn(a, 127.0) : INFINITY;
        __syncthreads();
        if (!good) {
            if (tid == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
        } else if (tid < 64 && h0 * D + tid * 4 < p.Hkv * D) {
            *reinterpret_cast<uint32_t*>(p.mean + ((size_t)first * p.Hkv + h0) * D + tid * 4) = *reinterpret_cast<const uint32_t*>(s_out + tid * 4);
        }
    }
}

// ------------------------------------------------------------------------------------------------ selection
constexpr int kSelThreads = 256, kSelQueries = 32;            // queries of a tile

struct SelectParams {
    const __nv_bfloat16* q;
    const int32_t *q_start, *n_nodes;
    const int8_t* mean;
    const float* scale;
    const int32_t *table, *ctx_len;
    int32_t* out;
    int B, T, Hq, Hkv, G, P, max_pages, num_pages, n_rows, max_chunk, max_ctx;
    int shift, K, n_first, n_last;
    uint32_t* status;
};

__device__ __forceinline__ uint32_t score_key(int dot, float scale) {
    float s = __int2float_rn(dot) * scale;
    if (s != s) return 0xFFFFFFFFu;                           // not a number: before all others
    if (s == 0.f) s = 0.f;                                    // -0 is 0
    const uint32_t u = __float_as_uint(s);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

template <int D>
__global__ void __launch_bounds__(kSelThreads) cb_block_select_kernel(const SelectParams p) {
    extern __shared__ uint32_t s_key[];                       // [blocks]: largest products, then the scores' keys
    __shared__ __align__(16) int8_t s_q[kSelQueries][D];
    __shared__ uint32_t s_hist[256], s_warp[8], s_eq[8], s_pick[2];
    CB_PDL_ENTRY();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int kh = blockIdx.x % p.Hkv, b = blockIdx.x / p.Hkv;
    int32_t* const out = p.out + (size_t)blockIdx.x * p.K;
    // the rows, and whether they and the context are what the call says
    int row0, n, error = 0;
    if (p.q_start) {
        row0 = p.q_start[b];
        const int end = p.q_start[b + 1];
        n = end - row0;
        if (n != 0 && (row0 < 0 || end < row0 || end > p.n_rows || n > p.max_chunk)) error = CB_ERR_INVALID_ARG;
    } else {
        row0 = b * p.T;
        n = p.n_nodes[b];
        if (n < 0 || n > p.T) error = CB_ERR_INVALID_ARG;
    }
    const int ctx = p.ctx_len[b];
    if (!error && n != 0) error = ctx < 0 ? CB_ERR_INVALID_ARG : (ctx > p.max_ctx ? CB_ERR_KV_FULL : 0);
    const int nb = error || n == 0 ? 0 : cb_blocks_of(ctx, p.shift);
    if (nb <= p.K) {                                          // all there are
        for (int k = tid; k < p.K; k += kSelThreads) out[k] = k < nb ? k : -1;
        if (error && tid == 0 && kh == 0) atomicCAS(p.status, 0u, (uint32_t)error);
        return;
    }
    const int nq = n * p.G;
    auto query = [&](int i) { return p.q + ((size_t)(row0 + i / p.G) * p.Hq + kh * p.G + i % p.G) * D; };
    // largest magnitude of the queries, as bits of bf16
    uint32_t top = 0;
    for (int k = tid; k < nq * (D / 8); k += kSelThreads) {
        const uint4 v = *reinterpret_cast<const uint4*>(query(k / (D / 8)) + k % (D / 8) * 8);
        top = __vmaxu2(top, __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)));
    }
    top = max(top & 0xFFFFu, top >> 16);
    top = __reduce_max_sync(CB_FULL, top);
    if (lane == 0) s_warp[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) top = max(top, s_warp[w]);
    const float r = __fdiv_rn(127.f, fmaxf(__uint_as_float(top << 16), 1e-30f));
    const int per = p.shift - 4;
    for (int q0 = 0; q0 < nq; q0 += kSelQueries) {
        const int nt = min(kSelQueries, nq - q0);
        __syncthreads();
        for (int k = tid; k < nt * (D / 8); k += kSelThreads) {
            const int i = k / (D / 8), c = k % (D / 8) * 8;
            const uint4 v = *reinterpret_cast<const uint4*>(query(q0 + i) + c);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s_q[i][c + 2 * e] = (int8_t)__float2int_rn(__uint_as_float(w[e] << 16) * r);
                s_q[i][c + 2 * e + 1] = (int8_t)__float2int_rn(__uint_as_float(w[e] & 0xFFFF0000u) * r);
            }
        }
        __syncthreads();
        for (int j = tid; j < nb; j += kSelThreads) {
            const int page = p.table[(size_t)b * p.max_pages + (j << per)];
            const bool good = page >= 0 && page < p.num_pages;
            uint4 m[D / 16];
            const uint4* src = reinterpret_cast<const uint4*>(p.mean + ((size_t)(good ? page : 0) * p.Hkv + kh) * D);
#pragma unroll
            for (int c = 0; c < D / 16; ++c) m[c] = src[c];
            int best = q0 == 0 ? INT32_MIN : (int)s_key[j];
            for (int i = 0; i < nt; ++i) {
                int dot = 0;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const uint4 q = *reinterpret_cast<const uint4*>(&s_q[i][c * 16]);
                    dot = __dp4a((int)m[c].x, (int)q.x, dot); dot = __dp4a((int)m[c].y, (int)q.y, dot);
                    dot = __dp4a((int)m[c].z, (int)q.z, dot); dot = __dp4a((int)m[c].w, (int)q.w, dot);
                }
                best = max(best, dot);
            }
            if (q0 + nt < nq) s_key[j] = (uint32_t)best;
            else {
                s_key[j] = score_key(best, good ? p.scale[(size_t)page * p.Hkv + kh] : 0.f);
                if (!good) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
            }
        }
    }
    // The want-th largest key of the candidates, eight bits at a time from the top: `prefix` with `left` of its equals wanted.
    const int lo = p.n_first, hi = nb - p.n_last;
    uint32_t prefix = 0, left = (uint32_t)(p.K - p.n_first - p.n_last);
    if (left > 0)
        for (int bits = 24; bits >= 0; bits -= 8) {
            s_hist[tid] = 0;
            __syncthreads();
            for (int j = lo + tid; j < hi; j += kSelThreads) {
                const uint32_t k = s_key[j];
                if (bits == 24 || (k >> (bits + 8)) == (prefix >> (bits + 8))) atomicAdd(&s_hist[(k >> bits) & 255u], 1u);
            }
            __syncthreads();
            if (warp == 0) {
                uint32_t c[8], sum = 0;                       // lane 0 has the largest digits
#pragma unroll
                for (int e = 0; e < 8; ++e) { c[e] = s_hist[255 - (lane * 8 + e)]; sum += c[e]; }
                uint32_t before = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(CB_FULL, before, o); if (lane >= o) before += y; }
                before -= sum;
                if (before < left && left <= before + sum) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (before < left && left <= before + c[e]) { s_pick[0] = prefix | ((uint32_t)(255 - (lane * 8 + e)) << bits); s_pick[1] = left - before; }
                        before += c[e];
                    }
                }
            }
            __syncthreads();
            prefix = s_pick[0]; left = s_pick[1];
        }
    else __syncthreads();
    const bool any = p.K > p.n_first + p.n_last;
    // In order: a run of blocks per thread, where its chosen ones go by the sums before it.
    const int run = (nb + kSelThreads - 1) / kSelThreads, j0 = min(tid * run, nb), j1 = min(j0 + run, nb);
    uint32_t gt = 0, eq = 0;
    for (int j = j0; j < j1; ++j) {
        const bool cand = j >= lo && j < hi;
        if (!cand) ++gt;
        else if (any) { gt += s_key[j] > prefix; eq += s_key[j] == prefix; }
    }
    uint32_t gs = gt, es = eq;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(CB_FULL, gs, o), z = __shfl_up_sync(CB_FULL, es, o);
        if (lane >= o) { gs += y; es += z; }
    }
    if (lane == 31) { s_warp[warp] = gs; s_eq[warp] = es; }
    __syncthreads();
    gs -= gt; es -= eq;
    for (int w = 0; w < warp; ++w) { gs += s_warp[w]; es += s_eq[w]; }
    for (int j = j0; j < j1; ++j) {
        const bool cand = j >= lo && j < hi;
        const bool over = !cand || (any && s_key[j] > prefix), equal = cand && any && s_key[j] == prefix;
        if (over || (equal && es < left)) out[gs + min(es, left)] = j;
        gs += over; es += equal;
    }
}

std::mutex g_mutex;
size_t g_smem[2][64];

}  // namespace

extern "C" cb_status cb_block_summary(cb_ctx* ctx, const cb_block_summary_args* a, void* stream) {
    CB_CHECK_ARG(ctx && a);
    CB_CHECK_ARG(a->k_pool && a->block_table && a->from_len && a->to_len && a->k_mean && a->k_scale && a->max_pages >= 1 && a->num_pages >= 1);
    CB_CHECK_ARG(a->block == 16 || a->block == 32 || a->block == 64 || a->block == 128);
    CB_CHECK_ARG((((uintptr_t)a->k_pool | (uintptr_t)a->k_mean) & 15) == 0 && ((uintptr_t)a->k_scale & 3) == 0);
    const cb_config& c = ctx->cfg;
    if (c.page_size != 16 || c.batch > CB_MAX_ASSIGN) return CB_ERR_UNSUPPORTED;
    SummaryParams p = {};
    p.k_pool = (const __nv_bfloat16*)a->k_pool; p.table = a->block_table; p.from = a->from_len; p.to = a->to_len;
    p.mean = a->k_mean; p.scale = a->k_scale;
    p.B = c.batch; p.Hkv = c.n_kv_heads; p.P = c.page_size; p.max_pages = a->max_pages; p.num_pages = a->num_pages;
    p.status = ctx->d_status;
    const size_t smem = (size_t)c.batch * 8;
    const auto launch = [&](auto kernel) -> cb_status {
        if (smem > 16 * 1024) CB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, CB_MAX_ASSIGN * 8));
        CB_CUDA(cb_launch_pdl(kernel, dim3(ctx->num_sms * 4), dim3(kSumThreads), smem, (cudaStream_t)stream, p));
        cb_count_launch(1);
        return CB_OK;
    };
    const auto by_block = [&](auto d) -> cb_status {
        constexpr int D = decltype(d)::value;
        switch (a->block) {
            case 16: return launch(cb_block_summary_kernel<D, 16>);
            case 32: return launch(cb_block_summary_kernel<D, 32>);
            case 64: return launch(cb_block_summary_kernel<D, 64>);
            default: return launch(cb_block_summary_kernel<D, 128>);
        }
    };
    return c.head_dim == 128 ? by_block(std::integral_constant<int, 128>{}) : by_block(std::integral_constant<int, 64>{});
}

extern "C" cb_status cb_block_select(cb_ctx* ctx, const cb_block_select_args* a, void* stream) {
    CB_CHECK_ARG(ctx && a);
    CB_CHECK_ARG((a->q_start != nullptr) != (a->n_nodes != nullptr));
    CB_CHECK_ARG(a->k_mean && a->k_scale && a->block_table && a->ctx_len && a->blocks && a->max_pages >= 1 && a->num_pages >= 1);
    CB_CHECK_ARG(a->block == 16 || a->block == 32 || a->block == 64 || a->block == 128);
    CB_CHECK_ARG(a->n_rows >= 0 && a->max_chunk >= 0 && a->max_ctx >= 0 && (a->q || (a->q_start && a->n_rows == 0)));
    CB_CHECK_ARG(a->n_first >= 0 && a->n_last >= 1 && a->n_select <= CB_MAX_SELECT && a->n_first <= a->n_select - a->n_last);
    CB_CHECK_ARG((((uintptr_t)a->q | (uintptr_t)a->k_mean) & 15) == 0 && ((uintptr_t)a->k_scale & 3) == 0);
    const cb_config& c = ctx->cfg;
    if (c.page_size != 16) return CB_ERR_UNSUPPORTED;
    SelectParams p = {};
    p.q = (const __nv_bfloat16*)a->q; p.q_start = a->q_start; p.n_nodes = a->n_nodes; p.mean = a->k_mean; p.scale = a->k_scale;
    p.table = a->block_table; p.ctx_len = a->ctx_len; p.out = a->blocks;
    p.B = c.batch; p.T = c.max_nodes; p.Hq = c.n_q_heads; p.Hkv = c.n_kv_heads; p.G = c.n_q_heads / c.n_kv_heads; p.P = c.page_size;
    p.max_pages = a->max_pages; p.num_pages = a->num_pages; p.n_rows = a->n_rows;
    p.max_chunk = a->max_chunk > 0 ? std::min(a->max_chunk, a->n_rows) : a->n_rows;
    const long long cap = std::min<long long>((long long)a->max_pages * c.page_size, 1ll << 30);
    p.max_ctx = (int)(a->max_ctx > 0 ? std::min<long long>(a->max_ctx, cap) : cap);
    p.shift = __builtin_ctz((unsigned)a->block); p.K = a->n_select; p.n_first = a->n_first; p.n_last = a->n_last;
    p.status = ctx->d_status;
    const int blocks = cb_blocks_of(p.max_ctx, p.shift);
    if (blocks > 32768) return CB_ERR_UNSUPPORTED;
    const size_t smem = (size_t)blocks * 4;
    const auto launch = [&](auto kernel, int which) -> cb_status {
        {
            std::lock_guard<std::mutex> lock(g_mutex);
            size_t fresh = 0;
            CB_CUDA(cb_allow_smem(kernel, smem, ctx->device >= 0 && ctx->device < 64 ? &g_smem[which][ctx->device] : &fresh));
        }
        CB_CUDA(cb_launch_pdl(kernel, dim3(p.B * p.Hkv), dim3(kSelThreads), smem, (cudaStream_t)stream, p));
        cb_count_launch(1);
        return CB_OK;
    };
    return c.head_dim == 128 ? launch(cb_block_select_kernel<128>, 1) : launch(cb_block_select_kernel<64>, 0);
}
