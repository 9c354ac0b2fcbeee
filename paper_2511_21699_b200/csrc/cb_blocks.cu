// Block summaries and the selection of blocks by them.
//
// cb_block_summary.  The mean of a block's keys, in 64 bits: a sum of up to 128 bf16 values is exact there (8-bit mantissas) while their exponents lie no more than 38 apart, and
// beyond that its bits follow from the order, which is always the same (a warp takes every eighth token, the warps are added up in turn).  So a block may be summarised token by
// token or all at once, and the bits are the same.  A CTA takes
// a block and 256 channels (two heads of 128 or four of 64): its eight warps take every eighth token, 512 contiguous bytes of it each, all of a warp's
// loads under way at once, the next block's while this one's sums are put together in shared memory, where a thread finishes a channel.  Issue slots bound it, 64% of
// them busy: 26.5 us for 100 MB of keys (8 heads of 128, blocks of 64), 3.8 TB/s; the block of one new token in each of 64 sequences 8 us from a cold start.
//
// cb_block_select.  A CTA, or a cluster of up to eight where there are few, per (sequence, kv head).  The queries become whole numbers of a common scale, the
// summaries are whole numbers already, so that the scores are exact and the choice is the same however the work is cut.  64 single tokens over 1 k to 32 k tokens in blocks of
// 64, 8 kv heads: 11.4 us, most of it the longest unit's chain (lengths and pages, summaries, scores, search); the 19 MB take 2.8.
#include <algorithm>
#include <mutex>

#include "cb_scan.cuh"
#include "cb_select.cuh"

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

// A bf16, the upper half of a word, as a double 2^-896 times as large: sign, exponent and mantissa moved to their places, which does for zero and
// the smallest numbers too (infinity and NaN become numbers and are looked for apart).
__device__ __forceinline__ double small_double(uint32_t upper) { return __hiloint2double(((int)upper >> 3) & 0x8FFFE000, 0); }
constexpr double kSmallDouble = 0x1p896;

template <int D, int S>
__global__ void __launch_bounds__(kSumThreads, S == 128 ? 2 : 3) cb_block_summary_kernel(const SummaryParams p) {
    constexpr int HG = 256 / D, LH = D / 8, WH = D / 32, T = S / 8;   // heads of a CTA, lanes of a head that load, its warps that finish it, tokens of a warp
    constexpr int ROW = 34;                                   // channel lane * 8 + e lies at e * ROW + lane: no bank twice, written or read
    extern __shared__ uint32_t s_sums[];                      // [B]
    __shared__ uint32_t s_scratch[kSumThreads / 32];
    __shared__ double s_part[8][8 * ROW];                     // the warps' sums
    __shared__ uint32_t s_bad[8];                             // of a warp's tokens: heads with a number that is not finite
    __shared__ uint2 s_top[8];
    __shared__ __align__(16) int8_t s_out[256];
    CB_PDL_ENTRY();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int error = 0;
    cb_block_sums<kSumThreads, 1>(p.B, s_sums, s_scratch, [&](int b, uint32_t* blocks) {
        const int lo = p.from[b], hi = p.to[b];
        if (lo >= hi) return;
        if (lo < 0) error = CB_ERR_INVALID_ARG;
        else if (hi > (long long)p.max_pages * p.P) error = CB_ERR_KV_FULL;
        else *blocks = (uint32_t)((hi - 1) / S - lo / S + 1);
    });
    if (error && blockIdx.x == 0) atomicCAS(p.status, 0u, (uint32_t)error);
    // Items: a block's 256 channels from head h0 on, all groups of heads of one block after the other, dealt to the CTAs in turn.
    const uint32_t blocks = s_sums[p.B - 1], groups = (uint32_t)(p.Hkv + HG - 1) / HG, step_at = gridDim.x / groups, step_group = gridDim.x % groups;
    struct Place { uint32_t at, group; };
    auto after = [&](Place x) {
        x.at += step_at; x.group += step_group;
        if (x.group >= groups) { x.group -= groups; ++x.at; }
        return x;
    };
    struct Item { int h0, n, page; };                         // lane l has its l-th page; n: tokens, 0 if there is no such item
    auto locate = [&](Place x) {
        Item i = {0, 0, 0};
        if (x.at >= blocks) return i;
        i.h0 = (int)x.group * HG;
        const int b = cb_upper(s_sums, p.B, x.at);
        const int blk = p.from[b] / S + (int)(x.at - (b > 0 ? s_sums[b - 1] : 0u));
        i.n = min(S, p.to[b] - blk * S);
        if (lane < (i.n + 15) / 16) i.page = p.table[(size_t)b * p.max_pages + blk * (S / 16) + lane];
        return i;
    };
    uint4 v[T];
    // All loads of an item at once.  False: a page outside the pool.
    auto issue = [&](const Item& i) {
        const bool good = __all_sync(CB_FULL, i.page >= 0 && i.page < p.num_pages);
        const int head = i.h0 + lane / LH, n = good && head < p.Hkv ? i.n : 0;
        // token warp + 8 k of the block is row warp + 8 (k & 1) of its page k / 2
        const __nv_bfloat16* const at = p.k_pool + ((size_t)warp * p.Hkv + head) * D + (lane % LH) * 8;
        const size_t row = (size_t)p.Hkv * D;
#pragma unroll
        for (int k = 0; k < T; k += 2) {
            const __nv_bfloat16* src = at + (size_t)__shfl_sync(CB_FULL, i.page, k >> 1) * (16 * row);
            v[k] = v[k + 1] = make_uint4(0, 0, 0, 0);
            if (warp + 8 * k < n) v[k] = *reinterpret_cast<const uint4*>(src);
            if (warp + 8 * k + 8 < n) v[k + 1] = *reinterpret_cast<const uint4*>(src + 8 * row);
        }
        return good;
    };
    Place place = {blockIdx.x / groups, blockIdx.x % groups};
    Item now = locate(place);
    bool good = issue(now);
    place = after(place);
    Item next = locate(place);
    while (now.n > 0) {
        // A word's lower number by a conversion, its upper one by moving bits: half of the numbers to either pipe, both of which are slow (16 conversions, or 64
        // operations at two to three a number, a cycle and SM; memory brings 12 numbers a cycle).
        double sum[8] = {};
        __nv_bfloat162 most = __float2bfloat162_rn(0.f);      // largest magnitudes, NaN above all
#pragma unroll
        for (int k = 0; k < T; ++k) {
            const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum[2 * e] += (double)__uint_as_float(w[e] << 16);
                sum[2 * e + 1] += small_double(w[e]);
                most = __hmax2_nan(most, __habs2(reinterpret_cast<const __nv_bfloat162&>(w[e])));
            }
        }
        // the next item's keys are on their way while this one's sums are put together
        const Item it = now;
        const bool it_good = good;
        now = next;
        good = issue(now);
        place = after(place);
        next = locate(place);
#pragma unroll
        for (int e = 0; e < 8; ++e) s_part[warp][e * ROW + lane] = sum[e];
        const uint32_t bits = reinterpret_cast<const uint32_t&>(most) & 0x7FFF7FFFu;
        const uint32_t bad = __ballot_sync(CB_FULL, max(bits & 0xFFFFu, bits >> 16) >= 0x7F80u);
        if (lane == 0) s_bad[warp] = bad;
        __syncthreads();
        // a channel per thread: its mean, and the largest magnitude of its head's
        double m = 0.0;
        uint32_t any_bad = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) { m += s_part[w][(tid & 7) * ROW + (tid >> 3)]; any_bad |= s_bad[w]; }
        if (tid & 1) m *= kSmallDouble;
        m = it.n == S ? m * (1.0 / S) : __ddiv_rn(m, (double)it.n);   // (the same: S is a power of two)
        const int group = tid / D;
        const bool finite = (any_bad >> (group * LH) & (uint32_t)((1ull << LH) - 1ull)) == 0u;
        const uint32_t hi = (uint32_t)__double2hiint(m) & 0x7FFFFFFFu, lo = (uint32_t)__double2loint(m);
        const uint32_t top_hi = __reduce_max_sync(CB_FULL, hi), top_lo = __reduce_max_sync(CB_FULL, hi == top_hi ? lo : 0u);
        if (lane == 0) s_top[warp] = make_uint2(top_hi, top_lo);
        __syncthreads();
        uint2 top = make_uint2(0u, 0u);
#pragma unroll
        for (int w = 0; w < WH; ++w) {
            const uint2 x = s_top[group * WH + w];
            if (x.x > top.x || (x.x == top.x && x.y > top.y)) top = x;
        }
        const double a = __hiloint2double((int)top.x, (int)top.y);
        // The whole number by a quotient in 32 bits, off by less than 127 * 2^-21, unless that lies near half way between two; then by the one in 64.
        const float f = __fdividef((float)m * 127.f, (float)a), whole = rintf(f);
        int q = (int)whole;
        if (!(fabsf(fabsf(f - whole) - 0.5f) > 0.001f) || !(a > 1e-30 && a < 1e36)) q = __double2int_rn(__ddiv_rn(__dmul_rn(m, 127.0), fmax(a, 1e-30)));
        s_out[tid] = finite ? (int8_t)q : (int8_t)0;
        const int first = __shfl_sync(CB_FULL, it.page, 0);
        if (it_good && tid % D == 0 && it.h0 + group < p.Hkv) p.scale[(size_t)first * p.Hkv + it.h0 + group] = finite ? (float)__ddiv_rn(a, 127.0) : INFINITY;
        __syncthreads();
        if (!it_good) {
            if (tid == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
        } else if (tid < 64 && it.h0 * D + tid * 4 < p.Hkv * D) {
            *reinterpret_cast<uint32_t*>(p.mean + ((size_t)first * p.Hkv + it.h0) * D + tid * 4) = *reinterpret_cast<const uint32_t*>(s_out + tid * 4);
        }
    }
}

// ------------------------------------------------------------------------------------------------ selection by few queries
// A warp takes 16 blocks at a time and has three such steps under way.  Four CTAs an SM, so that 592 units are resident at once (with 32 blocks in two steps, three
// CTAs an SM, 68 of 512 units came in a second wave).  That many fit while the keys of all blocks that max_ctx allows take what the rings leave: up to 1,260 blocks
// with 128 dims and 7,404 with 64; three up to 6,124 and 12,268.
constexpr int kFewThreads = 256, kFewRows = 16, kFewStages = 3, kFewStep = kFewThreads / 32 * kFewRows;
template <int D> constexpr int kFewWarpBytes = kFewStages * kFewRows * (D + 4);   // summaries and scales

__device__ __forceinline__ void mma_s8(int* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Up to NT x 8 queries, single tokens mostly: memory's round trips are what a launch takes, so all that can be asked for at once is.  A warp's queries are its
// own (a row of 8 lies in the registers of 32 lanes as the products take it), its 16 blocks' summaries come by asynchronous copies.
//
// The products are m16n8k32 of bytes, 16 blocks by 8 queries by 32 dims (tcgen05's smallest tile of 128 blocks would wait for four warps' copies, for no gain: the
// pipe is 2% busy).  A dot product does not mind the order of its terms, so the k-th step takes, of the 16-byte pieces that lane t of a row's four lanes holds
// (piece t, and with 128 dims piece t + 4), the words that make a fragment: both sides come from memory in 16-byte pieces and go into the products as they are.
template <int D, int NT>
__global__ void __launch_bounds__(kFewThreads, 4) cb_select_few_kernel(const CbSelectParams p) {
    constexpr int W = D / 16, L = D / 16;                     // words of a row that a lane holds; lanes that copy a row
    extern __shared__ __align__(16) uint32_t s_dyn[];
    __shared__ __align__(16) uint32_t s_scratch[cb_pick_words<kFewThreads>];
    uint32_t* const s_key = s_dyn;
    CB_PDL_ENTRY();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    uint8_t* const s_rows = reinterpret_cast<uint8_t*>(s_dyn + p.key_words) + warp * kFewWarpBytes<D>;
    float* const s_scale = reinterpret_cast<float*>(s_rows + kFewStages * kFewRows * D);
    uint32_t rank, ranks;
    asm("mov.u32 %0, %cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %cluster_nctarank;" : "=r"(ranks));
    const int unit = blockIdx.x / ranks;
    const int step = (int)ranks * kFewStep, start = (int)rank * kFewStep + warp * kFewRows;
    // A block's first page; lanes l and l + 16 have block l of the warp's 16.  Asked for beside the lengths, as far as the table has columns; a block behind the context
    // is not used.
    const int32_t* const table = p.table + (size_t)(unit / p.Hkv) * p.max_pages;
    auto page_of = [&](int base) {
        const long long col = (long long)(base + (lane & 15)) << (p.shift - 4);
        return col < p.max_pages ? table[col] : -1;
    };
    int pages[kFewStages];
#pragma unroll
    for (int k = 0; k < kFewStages; ++k) pages[k] = page_of(start + k * step);
    int page_next = page_of(start + kFewStages * step);
    const CbSelectUnit u = cb_select_unit(p, unit, rank == 0, tid, kFewThreads);
    const int nb = u.nb, nq = u.n * p.G;
    if (nb == 0) return;
    for (int k = tid; k < cb_pick_words<kFewThreads>; k += kFewThreads) s_scratch[k] = 0u;
    if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    // Row i's piece c lies at piece c ^ (i & 1) * 4 (128 dims), so that eight lanes that read two rows meet no bank twice.
    auto piece = [&](int stage, int i, int c) { return s_rows + (stage * kFewRows + i) * D + ((D == 128 ? c ^ ((i & 1) << 2) : c) << 4); };
    // The 16 blocks from base on into a stage; a page outside the pool has the scale 0.
    auto load_rows = [&](int base, int stage, int page) {
        if (base < nb) {
            const int j = base + (lane & 15);
            const bool good = j < nb && page >= 0 && page < p.num_pages;
            const int at = good ? page : 0;
#pragma unroll
            for (int k = 0; k < kFewRows * L / 32; ++k) {
                const int row = k * (32 / L) + lane / L, pg = __shfl_sync(CB_FULL, at, row);
                const int8_t* src = p.mean + ((size_t)pg * p.Hkv + u.kh) * D + lane % L * 16;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(piece(stage, row, lane % L))), "l"(src) : "memory");
            }
            if (lane < 16) {
                float* const to = s_scale + stage * kFewRows + lane;
                if (good) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(p.scale + (size_t)at * p.Hkv + u.kh) : "memory");
                else {
                    *to = 0.f;
                    if (j < nb) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < kFewStages; ++k) load_rows(start + k * step, k, pages[k]);
    // the queries: each one's pieces tig and tig + 4, whole numbers of a common scale; what there is less than 8 is filled up with the first
    uint32_t w[NT][W], top = 0;
    {
        uint4 v[NT][W / 2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const __nv_bfloat16* src = cb_select_query<D>(p, u, t * 8 + gid < nq ? t * 8 + gid : 0) + tig * 16;
#pragma unroll
            for (int c = 0; c < W / 2; ++c) v[t][c] = *reinterpret_cast<const uint4*>(src + (c >> 1) * 64 + (c & 1) * 8);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < W / 2; ++c) top = cb_max_bits(top, v[t][c]);
        top = __reduce_max_sync(CB_FULL, max(top & 0xFFFFu, top >> 16));
        const float r = cb_whole_factor(top);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < W / 2; ++c) { const uint2 x = cb_whole8(v[t][c], r); w[t][2 * c] = x.x; w[t][2 * c + 1] = x.y; }
    }
    uint32_t key0 = 0;                                        // the first CTA's keys, which all of a cluster write to
    if (ranks > 1) {
        key0 = cb_cluster_first(s_key);
        cb_cluster_wait();
    }
    int stage = 0;
    for (int base = start; base < nb; base += step) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 1) : "memory");
        __syncwarp();
        uint32_t a[2][W];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < W / 4; ++c) {
                const uint4 x = *reinterpret_cast<const uint4*>(piece(stage, h * 8 + gid, tig + 4 * c));
                a[h][4 * c] = x.x; a[h][4 * c + 1] = x.y; a[h][4 * c + 2] = x.z; a[h][4 * c + 3] = x.w;
            }
        const float scale = s_scale[stage * kFewRows + (lane & 15)];
        __syncwarp();                                         // the stage has been read
        load_rows(base + kFewStages * step, stage, page_next);
        page_next = page_of(base + (kFewStages + 1) * step);
        int best[2] = {INT32_MIN, INT32_MIN};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            int c[4] = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < W / 2; ++s) mma_s8(c, a[0][s], a[1][s], a[0][s + W / 2], a[1][s + W / 2], w[t][s], w[t][s + W / 2]);
            best[0] = max(best[0], max(c[0], c[1]));
            best[1] = max(best[1], max(c[2], c[3]));
        }
        int mine = 0;                                         // lane l < 16: the largest product of block base + l
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int v = best[h];
            v = max(v, __shfl_xor_sync(CB_FULL, v, 1));
            v = max(v, __shfl_xor_sync(CB_FULL, v, 2));
            v = __shfl_sync(CB_FULL, v, (lane & 7) * 4);
            if (((lane >> 3) & 1) == h) mine = v;
        }
        const int j = base + lane;
        if (lane < 16 && j < nb) {
            const uint32_t key = cb_score_key(mine, scale);
            if (ranks > 1) cb_cluster_store(key0 + 4u * (uint32_t)j, key);
            else s_key[j] = key;
        }
        __syncwarp();
        stage = stage == kFewStages - 1 ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (ranks > 1) {
        cb_cluster_arrive();
        cb_cluster_wait();
        if (rank != 0) return;
    }
    __syncthreads();
    cb_pick<kFewThreads>(p, nb, s_key, s_scratch, p.out + (size_t)unit * p.K);
}

std::mutex g_mutex;
size_t g_smem[4][64];

}  // namespace

extern "C" cb_status cb_block_summary(cb_ctx* ctx, const cb_block_summary_args* a, void* stream) {
    CB_CHECK_ARG(ctx && a);
    CB_CHECK_ARG(a->k_pool && a->block_table && a->from_len && a->to_len && a->k_mean && a->k_scale && a->max_pages >= 1 && a->num_pages >= 1);
    CB_CHECK_ARG(a->block == 16 || a->block == 32 || a->block == 64 || a->block == 128);
    CB_CHECK_ARG((((uintptr_t)a->k_pool | (uintptr_t)a->k_mean) & 15) == 0 && ((uintptr_t)a->k_scale & 3) == 0);
    const cb_config& c = ctx->cfg;
    if (c.batch > CB_MAX_ASSIGN) return CB_ERR_UNSUPPORTED;
    if ((long long)c.batch * (((long long)a->max_pages * c.page_size + a->block - 1) / a->block) >= (long long)CB_SUM_CAP) return CB_ERR_UNSUPPORTED;   // (blocks are counted up to there)
    SummaryParams p = {};
    p.k_pool = (const __nv_bfloat16*)a->k_pool; p.table = a->block_table; p.from = a->from_len; p.to = a->to_len;
    p.mean = a->k_mean; p.scale = a->k_scale;
    p.B = c.batch; p.Hkv = c.n_kv_heads; p.P = c.page_size; p.max_pages = a->max_pages; p.num_pages = a->num_pages;
    p.status = ctx->d_status;
    const size_t smem = (size_t)c.batch * 4;
    const auto launch = [&](auto kernel) -> cb_status {
        if (smem > 16 * 1024) CB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, CB_MAX_ASSIGN * 4));
        CB_CUDA(cb_launch_pdl(kernel, dim3(ctx->num_sms * (a->block == 128 ? 2 : 3)), dim3(kSumThreads), smem, (cudaStream_t)stream, p));
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
    CB_CHECK_ARG(a->n_first >= 0 && a->n_last >= 1 && a->n_select >= 1 && a->n_select <= CB_MAX_SELECT && a->n_first <= a->n_select - a->n_last);
    CB_CHECK_ARG((((uintptr_t)a->q | (uintptr_t)a->k_mean) & 15) == 0 && ((uintptr_t)a->k_scale & 3) == 0);
    const cb_config& c = ctx->cfg;
    CbSelectParams p = {};
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
    if (blocks > 16384) return CB_ERR_UNSUPPORTED;            // (keys of all blocks beside the tiles in shared memory)
    p.key_words = (blocks + 3) & ~3;
    p.g_inv = p.G > 1 ? 0xFFFFFFFFu / (uint32_t)p.G + 1u : 0u;
    // Row and head of a chunk's query x are exact while x times what g_inv is too large by stays below 2^32; longer chunks are turned away with those above the caller's bound.
    const uint32_t over = p.g_inv * (uint32_t)p.G;            // G g_inv - 2^32, less than G
    if (over) p.max_chunk = std::min(p.max_chunk, (int)std::min<uint32_t>(0xFFFFFFFFu / over / (uint32_t)p.G, INT32_MAX));
    if (!p.q_start && (long long)p.B * p.T > 0x7FFFFFFFll) return CB_ERR_UNSUPPORTED;
    // Up to 16 queries (rows x heads of the group) lie in a warp's registers, the others are for the tensor pipe, and 128 blocks a tile.  (8 kv heads of 128; 64 sequences of 1 k to
    // 32 k tokens in blocks of 64: 8 queries 10.0 and 33.5 us, 16 12.1 and 33.8; one of 32 k: 4.4 and 8.8, 5.2 and 8.8.  There are no forms for more queries than that; trial ones
    // for 24 and 32 took 14.1 and 17.3 us against 33.9, and 5.6 and 6.4 against 8.9.)  With few units a
    // cluster shares each one's blocks: as many CTAs as there are SMs for and tiles to keep them busy.  (Single tokens, 8 kv heads, 1, 2, 4 and 8 CTAs a unit: one
    // sequence of 8 k tokens 4.0, 4.3, 4.2, 4.4 us, of 32 k 6.0, 5.3, 4.8, 4.8, of 128 k 17.5, 13.6, 11.6, 10.5; eight of 128 k 18.5, 14.4, 15.5, 17.9; 18 of 32 k 6.4, 6.6, 8.8, 13.4.
    // Parts of 32 rows, where a CTA fills an SM: eight of 32 k 10.7, 10.2, 19.0, 41; twelve 10.8, 19.5, 27.8, 57.)
    const long long votes = (long long)(a->q_start ? p.max_chunk : p.T) * p.G;
    const int nt = votes <= 8 ? 1 : (votes <= 16 ? 2 : 0);
    int ctas = 1;
    while (ctas < 8 && (long long)p.B * p.Hkv * ctas * 2 <= ctx->num_sms && blocks > ctas * 128) ctas *= 2;
    if (nt == 0) return cb_select_launch_many(ctx, p, ctas, (cudaStream_t)stream);
    const size_t smem = (size_t)p.key_words * 4 + (size_t)(kFewThreads / 32) * (c.head_dim == 128 ? kFewWarpBytes<128> : kFewWarpBytes<64>);
    const auto launch = [&](auto kernel, int which) -> cb_status {
        {
            std::lock_guard<std::mutex> lock(g_mutex);
            size_t fresh = 0;
            CB_CUDA(cb_allow_smem(kernel, smem, ctx->device >= 0 && ctx->device < 64 ? &g_smem[which][ctx->device] : &fresh));
        }
        CB_CUDA(cb_launch_clusters(kernel, (unsigned)((long long)p.B * p.Hkv * ctas), (unsigned)ctas, kFewThreads, smem, (cudaStream_t)stream, p));
        cb_count_launch(1);
        return CB_OK;
    };
    if (c.head_dim == 128) return nt == 1 ? launch(cb_select_few_kernel<128, 1>, 0) : launch(cb_select_few_kernel<128, 2>, 1);
    return nt == 1 ? launch(cb_select_few_kernel<64, 1>, 2) : launch(cb_select_few_kernel<64, 2>, 3);
}
