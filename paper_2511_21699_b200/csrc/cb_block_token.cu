// Attention over selected blocks for few rows a unit: single tokens, up to 16 rows x heads of a kv head's group.
//
// Such a unit is a stream: two flops a byte and row.  (A tcgen05 tile has 128 rows, of which a token fills 1 to 16; chunk attention's kernel takes such units too, with
// a schedule, a ring and an epilogue made for tiles: 13.9 us for one token and 110 for 64 with lists of 2,048 tokens, 8 kv heads of 128, where this one takes 6.6 and 84, 95% of the copy
// rate.)  So here a warp works for itself: it has a ring of its own that an
// asynchronous copy fills with a page of keys and values at a time, m16n8k16 products with the keys (then the values' columns) as the 16 rows and the queries as
// the 8 columns, and its own running softmax.  Nobody waits for anybody until the end, where the block's warps, and a cluster's blocks through distributed shared
// memory, put their parts together.
//
//   S^T = K Q^T   16 keys x 8 queries: K's fragments by ldmatrix, the queries' stay in registers
//   P^T           in the same places; movmatrix turns each 8 x 8 of it into the next product's other operand
//   O^T += V^T P^T   16 columns x 8 queries: V's fragments by ldmatrix with transposition
//
// The reference maximum is moved only where a score lies 2^8 above it (a vote a page, no reduction); P is rounded to bf16 for its product (2^-8 of each at
// most), its sum is of the values before that.
#include <algorithm>

#include "cb_chunk_tc.cuh"

namespace {

// WARPS: 8 of two stages where all CTAs are resident at once, one an SM, and the launch is as long as its longest warp; 4 of three stages, two CTAs an SM, where there
// are more, and one's end should lie beside the middle of another.  (Stages of 8 KB with 128 dims; twice as many with 64.  64 sequences of 8 kv heads: 83 to 86 us with 4 warps of three
// stages, 86 of two, 90 with 8 of two; one sequence: 7.5 with 4, 6.7 with 8.)
template <int D, int NT, int WARPS_>
struct TokCfg {
    static constexpr int WARPS = WARPS_, THREADS = 32 * WARPS, STAGES = (WARPS == 8 ? 2 : 3) * (128 / D);
    static constexpr uint32_t PAGE = 16 * D * 2;              // a page's keys, or values, of one head
    static constexpr uint32_t WARP = STAGES * 2 * PAGE;
    static constexpr int ROWS = 8 * NT, STRIDE = D + 4;       // of a part's output in floats: eight columns of four queries meet no bank twice
    static constexpr uint32_t PART = ROWS * STRIDE * 4;       // fits the warp's ring
    static constexpr uint32_t OFF_BAR = WARPS * WARP, OFF_ML = OFF_BAR + (WARPS * STAGES * 8 + 15) / 16 * 16 + 16;   // [warps][rows] maximum, sum; abort flag before it
    static constexpr uint32_t OFF_GATHER = OFF_ML + WARPS * ROWS * 8;                                        // [cluster][rows][STRIDE], maximum and sum in the last places
    static_assert(PART <= WARP, "a warp's part lies in its ring");
};

__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t turn8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma_bf16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

struct TokMaps { CUtensorMap k, v; };

template <int D, int NT, int WARPS>
__global__ void __launch_bounds__(32 * WARPS) cb_block_token_kernel(const CbListParams p, const __grid_constant__ TokMaps maps) {
    using C = TokCfg<D, NT, WARPS>;
    extern __shared__ __align__(1024) uint8_t tok_smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    const uint32_t sbase = smem_u32(tok_smem);
    if (sbase & 1023u) {                                      // the swizzled pages need it; every thread sees the same address
        if (tid == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_UNSUPPORTED);
        return;
    }
    const uint32_t ring = sbase + warp * C::WARP, bars = sbase + C::OFF_BAR + warp * C::STAGES * 8;
    volatile int* const s_abort = reinterpret_cast<volatile int*>(tok_smem + C::OFF_ML - 16);
    float2* const s_ml = reinterpret_cast<float2*>(tok_smem + C::OFF_ML);
    float* const s_gather = reinterpret_cast<float*>(tok_smem + C::OFF_GATHER);
    uint32_t rank, ranks;
    asm("mov.u32 %0, %cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %cluster_nctarank;" : "=r"(ranks));
    if (lane == 0) {
        for (int s = 0; s < C::STAGES; ++s) mbar_init(bars + 8 * s, 1);
        if (warp == 0) { *s_abort = 0; tma_prefetch_desc(&maps.k); tma_prefetch_desc(&maps.v); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    CB_PDL_ENTRY();
    const int unit = blockIdx.x / ranks, b = unit / p.Hkv, kh = unit - b * p.Hkv;
    const CbChunkSeq s = cb_chunk_seq(p, b);
    if (s.n == 0) {
        if (s.error && rank == 0 && kh == 0 && tid == 0) atomicCAS(p.status, 0u, (uint32_t)s.error);
        return;
    }
    if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int nb = cb_blocks_of(p.ctx_len[b], p.l.shift), keys = s.ctx + s.n, all = (keys + 15) / 16;
    const int pg0 = (int)((long long)all * rank / ranks), pg1 = (int)((long long)all * (rank + 1) / ranks);
    const int count = pg1 - pg0 > warp ? (pg1 - pg0 - warp + WARPS - 1) / WARPS : 0;   // pages pg0 + warp, + WARPS, ...
    // Page numbers, a lane's of 32 pages at a time, the next 32 beside them: two dependent reads each.
    auto page_of = [&](int k) {
        int page = p.num_pages;                               // out of the pool: the copy fills zeros
        if (k < count) {
            const int col = cb_page_column(p.l, b, p.Hkv, kh, nb, pg0 + warp + k * WARPS);
            if ((uint32_t)col < (uint32_t)p.max_pages) page = p.block_table[(size_t)b * p.max_pages + col];
            if ((uint32_t)page >= (uint32_t)p.num_pages) page = p.num_pages;
        }
        return page;
    };
    int page_now = page_of(lane), page_later = page_of(32 + lane);
    auto fetch = [&](int k) {                                 // the warp's k-th page into its stage; page_now is that of its 32 or the 32 before
        const int page = __shfl_sync(CB_FULL, k & 32 ? page_later : page_now, k & 31);
        if (lane == 0) {
            const uint32_t st = k % C::STAGES, at = ring + st * 2 * C::PAGE;
            mbar_expect_tx(bars + 8 * st, 2 * C::PAGE);
            tma_load_5d(at, &maps.k, bars + 8 * st, 0, 0, 0, page * 2, kh);
            tma_load_5d(at + C::PAGE, &maps.v, bars + 8 * st, 0, 0, 0, page * 2, kh);
        }
        __syncwarp();
    };
    for (int k = 0; k < min(count, C::STAGES); ++k) fetch(k);
    // the queries' fragments: row r of the unit (token r / G, head r % G) is column r; what does not exist is zero
    const int rows = s.n * p.G;
    uint32_t q[NT][D / 16][2];
    int limit[NT][2];                                         // keys that this lane's columns of S^T see
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = t * 8 + gid, tok = (int)((uint32_t)r * p.g_inv >> 16);
        const __nv_bfloat16* src = p.q + ((size_t)(s.row0 + tok) * p.Hq + kh * p.G + r - tok * p.G) * D + tig * 2;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            q[t][d][0] = r < rows ? *reinterpret_cast<const uint32_t*>(src + d * 16) : 0u;
            q[t][d][1] = r < rows ? *reinterpret_cast<const uint32_t*>(src + d * 16 + 8) : 0u;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int x = t * 8 + tig * 2 + c;
            limit[t][c] = x < rows ? s.ctx + (int)((uint32_t)x * p.g_inv >> 16) + 1 : 0;
        }
    }
    float o[NT][D / 16][4] = {}, m[NT][2], l[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) { m[t][0] = m[t][1] = -INFINITY; l[t][0] = l[t][1] = 0.f; }
    // this lane's row and first 16-byte piece of the 8 x 8s that a fragment is made of
    const int krow = lane & 15, kpiece = lane >> 4, vrow = (lane & 7) + (lane >> 4) * 8, vpiece = (lane >> 3) & 1;
    auto at_piece = [&](uint32_t base, int row, int c) {      // groups of 8 keys; in each, 64-column blocks of 8 rows of 128 bytes, pieces swizzled
        return base + (row >> 3) * (D * 16) + (c >> 3) * 1024 + (row & 7) * 128 + (((c & 7) ^ (row & 7)) << 4);
    };
    bool ok = true;
    for (int k = 0; k < count; ++k) {
        const uint32_t st = k % C::STAGES, kb = ring + st * 2 * C::PAGE, vb = kb + C::PAGE;
        if (!(ok = __all_sync(CB_FULL, mbar_wait(bars + 8 * st, (k / C::STAGES) & 1, s_abort, p.status)))) break;   // (all lanes go on, or none)
        const int key0 = (pg0 + warp + k * WARPS) * 16;
        float sc[NT][4] = {};
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            uint32_t a[4];
            ldsm4(a, at_piece(kb, krow, d * 2 + kpiece));
#pragma unroll
            for (int t = 0; t < NT; ++t) mma_bf16(sc[t], a, q[t][d][0], q[t][d][1]);
        }
        const bool partial = key0 + 16 > s.ctx + 1;           // some rows may not see all of it
        bool move = false;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = sc[t][e] * p.scale_log2;
                if (partial && key0 + gid + (e >> 1) * 8 >= limit[t][e & 1]) x = -INFINITY;
                sc[t][e] = x;
                move |= !(x <= m[t][e & 1] + 8.f) && x != -INFINITY;
            }
        if (__any_sync(CB_FULL, move)) {
            // the columns' maxima over the page become the reference, where they are above it
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float mx = fmaxf(sc[t][c], sc[t][c + 2]);
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(CB_FULL, mx, x));
                    mx = fmaxf(mx, m[t][c]);
                    const float f = m[t][c] == -INFINITY ? 0.f : ex2(m[t][c] - mx);
                    m[t][c] = mx;
                    l[t][c] *= f;
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) { o[t][d][c] *= f; o[t][d][c + 2] *= f; }
                }
        }
        uint32_t pb[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = ex2(sc[t][e] - (m[t][e & 1] == -INFINITY ? 0.f : m[t][e & 1]));
            l[t][0] += w[0] + w[2]; l[t][1] += w[1] + w[3];
            pb[t][0] = turn8x8(pack_bf16(w[0], w[1])); pb[t][1] = turn8x8(pack_bf16(w[2], w[3]));
        }
        if (key0 + 16 > keys) {                               // slots behind the last token may hold anything: zeros, which NaN times zero is not
            for (int x = lane; x < (key0 + 16 - keys) * (D / 8); x += 32)
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at_piece(vb, keys - key0 + x / (D / 8), x % (D / 8))), "r"(0) : "memory");
            __syncwarp();
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            uint32_t a[4];
            ldsm4t(a, at_piece(vb, vrow, d * 2 + vpiece));
#pragma unroll
            for (int t = 0; t < NT; ++t) mma_bf16(o[t][d], a, pb[t][0], pb[t][1]);
        }
        __syncwarp();                                         // the stage has been read
        const int next = k + C::STAGES;
        if ((next & 31) == 0 && next > 0) {                   // on to the next 32 page numbers: the half that they are not in is free
            if (next & 32) page_now = page_of(next + 32 + lane);
            else page_later = page_of(next + 32 + lane);
        }
        if (next < count) fetch(next);
    }
    // ---- the warp's part into its ring, maxima and sums beside it
    __syncwarp();
    float* const part = reinterpret_cast<float*>(tok_smem + warp * C::WARP);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float sum = l[t][c];
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) sum += __shfl_xor_sync(CB_FULL, sum, x);
            const int r = t * 8 + tig * 2 + c;
            if (gid == 0) s_ml[warp * C::ROWS + r] = make_float2(m[t][c], sum);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                part[r * C::STRIDE + d * 16 + gid] = o[t][d][c];
                part[r * C::STRIDE + d * 16 + gid + 8] = o[t][d][c + 2];
            }
        }
    __syncthreads();
    if (ranks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // the first CTA is there
    // four columns of a row per thread: the warps' parts put together, and handed to the cluster's first CTA or written
    constexpr int QUADS = C::ROWS * (D / 4);
    auto put = [&](int r, int c, float4 v, float mx, float sum) {
        const int tok = (int)((uint32_t)r * p.g_inv >> 16);
        const size_t at = (size_t)(s.row0 + tok) * p.Hq + kh * p.G + r - tok * p.G;
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        *reinterpret_cast<uint2*>(p.out + at * D + c) = make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
        if (c == 0 && p.lse) p.lse[at] = (mx + log2f(sum)) * 0.6931471805599453f;
    };
    const uint32_t gather0 = ranks > 1 ? cluster_addr(smem_u32(s_gather), 0) + rank * (uint32_t)(C::ROWS * C::STRIDE * 4) : 0u;
    for (int x = tid; x < QUADS; x += C::THREADS) {
        const int r = x / (D / 4), c = x % (D / 4) * 4;
        if (r >= rows) break;
        float mx = -INFINITY, sum = 0.f;
        float2 ml[WARPS];
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { ml[w] = s_ml[w * C::ROWS + r]; mx = fmaxf(mx, ml[w].x); }
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = ml[w].x == -INFINITY ? 0.f : ex2(ml[w].x - mx);
            const float4 y = *reinterpret_cast<const float4*>(tok_smem + w * C::WARP + (r * C::STRIDE + c) * 4);
            sum = fmaf(f, ml[w].y, sum);
            v.x = fmaf(f, y.x, v.x); v.y = fmaf(f, y.y, v.y); v.z = fmaf(f, y.z, v.z); v.w = fmaf(f, y.w, v.w);
        }
        if (ranks == 1) put(r, c, v, mx, sum);
        else {
            const uint32_t at = gather0 + (uint32_t)(r * C::STRIDE) * 4u;
            asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at + 4u * c), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
            if (c == 0) asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at + 4u * D), "f"(mx), "f"(sum) : "memory");
        }
    }
    if (ranks > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (rank == 0)
            for (int x = tid; x < QUADS; x += C::THREADS) {
                const int r = x / (D / 4), c = x % (D / 4) * 4;
                if (r >= rows) break;
                float mx = -INFINITY, sum = 0.f;
                for (uint32_t k = 0; k < ranks; ++k) mx = fmaxf(mx, s_gather[(k * C::ROWS + r) * C::STRIDE + D]);
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                for (uint32_t k = 0; k < ranks; ++k) {
                    const float* g = s_gather + (k * C::ROWS + r) * C::STRIDE;
                    const float f = g[D] == -INFINITY ? 0.f : ex2(g[D] - mx);
                    const float4 y = *reinterpret_cast<const float4*>(g + c);
                    sum = fmaf(f, g[D + 1], sum);
                    v.x = fmaf(f, y.x, v.x); v.y = fmaf(f, y.y, v.y); v.z = fmaf(f, y.z, v.z); v.w = fmaf(f, y.w, v.w);
                }
                put(r, c, v, mx, sum);
            }
    }
    if (!ok || *s_abort)                                      // give copies that are still in flight time to land before the shared memory is released
        for (int k = 0; k < 64; ++k) __nanosleep(1000);
}

template <int D, int NT, int WARPS>
cb_status launch_token(const cb_ctx* ctx, const CbListParams& p, int ctas, cudaStream_t st) {
    using C = TokCfg<D, NT, WARPS>;
    static std::mutex mutex;
    static size_t have[kMaxDevices];
    const size_t smem = C::OFF_GATHER + (ctas > 1 ? (size_t)ctas * C::ROWS * C::STRIDE * 4 : 0);
    TokMaps maps;
    if (!encode_pool(&maps.k, p.k_pool, p) || !encode_pool(&maps.v, p.v_pool, p)) return CB_ERR_CUDA;
    {
        std::lock_guard<std::mutex> lock(mutex);
        size_t fresh = 0;
        CB_CUDA(cb_allow_smem(cb_block_token_kernel<D, NT, WARPS>, smem, ctx->device >= 0 && ctx->device < kMaxDevices ? &have[ctx->device] : &fresh));
    }
    CB_CUDA(cb_launch_clusters(cb_block_token_kernel<D, NT, WARPS>, (unsigned)((long long)p.B * p.Hkv * ctas), (unsigned)ctas, C::THREADS, smem, st, p, maps));
    cb_count_launch(1);
    return CB_OK;
}
template <int D, int NT>
cb_status launch_warps(const cb_ctx* ctx, const CbListParams& p, bool resident, int ctas, cudaStream_t st) {
    return resident ? launch_token<D, NT, 8>(ctx, p, ctas, st) : launch_token<D, NT, 4>(ctx, p, ctas, st);
}

}  // namespace

cb_status cb_block_launch_token(cb_ctx* ctx, const CbListParams& given, cudaStream_t st) {
    CbListParams p = given;
    if (p.num_pages >= 1 << 29) return CB_ERR_UNSUPPORTED;   // (a page's coordinate is twice its number)
    p.g_inv = 65536u / (uint32_t)p.G + 1u;                    // x / G = x * g_inv >> 16 for x < 256
    const long long units = (long long)p.B * p.Hkv, pages = (std::min<long long>(p.max_keys, ((long long)p.l.n_select << p.l.shift) + p.max_chunk) + 15) / 16;
    // A cluster shares a unit while all CTAs find an SM of their own and four pages each (8 sequences of 8 kv heads, 2,048 keys: 11.1 us with 128 CTAs, 14.3 with 64, 28 with
    // 512; 8 kv heads of one sequence, 512 keys: 5.1 us with 64 CTAs, 6.0 with 32).
    const bool resident = units <= ctx->num_sms;
    int ctas = 1;
    while (ctas < 8 && units * ctas * 2 <= ctx->num_sms && pages >= ctas * 2 * 4) ctas *= 2;
    const bool few = p.max_chunk * p.G <= 8;
    if (p.D == 128) return few ? launch_warps<128, 1>(ctx, p, resident, ctas, st) : launch_warps<128, 2>(ctx, p, resident, ctas, st);
    return few ? launch_warps<64, 1>(ctx, p, resident, ctas, st) : launch_warps<64, 2>(ctx, p, resident, ctas, st);
}
