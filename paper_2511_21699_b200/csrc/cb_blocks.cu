// Block summaries and the selection of blocks by them.
//
// cb_block_summary.  The mean of a block's keys, in 64 bits: a sum of up to 128 bf16 values is exact there (8-bit mantissas, unless exponents lie more than
// 2^38 apart), so a block's tokens may be dealt to warps, a block may be summarised token by token or all at once, and the bits are the same.  A CTA takes
// a block and 256 channels (two heads of 128 or four of 64): its eight warps take every eighth token, 512 contiguous bytes of it each, all of a warp's
// loads under way at once; the warps' sums are put together in shared memory, a channel per thread.  Memory bounds it: the keys are read once.
//
// cb_block_select.  A CTA, or a cluster of up to eight where there are few, per (sequence, kv head).  The queries become whole numbers of a common scale, the
// summaries are whole numbers already, so that the scores are exact and the choice is the same however the work is cut.
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
constexpr int kSelQueries = 512;                              // queries of a tile in shared memory

// Many queries are the tensor pipe's business (8 cycles a product) and need warps enough to feed it; of few there may be many units, and four CTAs an SM
// take 592 of them at once.
__host__ __device__ constexpr int sel_threads(int nt) { return nt ? 256 : 512; }

struct SelectParams {
    const __nv_bfloat16* q;
    const int32_t *q_start, *n_nodes;
    const int8_t* mean;
    const float* scale;
    const int32_t *table, *ctx_len;
    int32_t* out;
    int B, T, Hq, Hkv, G, P, max_pages, num_pages, n_rows, max_chunk, max_ctx;
    int shift, K, n_first, n_last;
    int key_words;            // words of the keys in shared memory; the queries lie behind them
    int tile;                 // queries that there is room for
    uint32_t* status;
};

__device__ __forceinline__ uint32_t score_key(int dot, float scale) {
    float s = __int2float_rn(dot) * scale;
    if (s != s) return 0xFFFFFFFFu;                           // not a number: before all others
    if (s == 0.f) s = 0.f;                                    // -0 is 0
    const uint32_t u = __float_as_uint(s);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ void mma_s8(int* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// NT: tiles of 8 queries that a warp keeps in registers; 0: any number, through shared memory.
//
// The products are m16n8k32 of bytes: 16 blocks by 8 queries by 32 dims.  A dot product does not mind the order of its terms, so the k-th step takes, of
// the 16-byte pieces that lane t of a row's four lanes holds (piece t, and with 128 dims piece t + 4), the words that make a fragment: rows are read from
// memory in 16-byte pieces and go into the products as they are.
template <int D, int NT>
__global__ void __launch_bounds__(sel_threads(NT), NT ? 4 : 1) cb_block_select_kernel(const SelectParams p) {
    constexpr int W = D / 16;                                 // words of a row that a lane holds
    constexpr int kThreads = sel_threads(NT), kWarps = kThreads / 32, kRows = kThreads;   // blocks that a CTA scores at a time: 32 a warp
    extern __shared__ __align__(16) uint32_t s_dyn[];
    __shared__ uint32_t s_hist[256], s_warp[kWarps], s_eq[kWarps], s_pick[3];
    uint32_t* const s_key = s_dyn;
    int8_t* const s_q = reinterpret_cast<int8_t*>(s_dyn + p.key_words);
    CB_PDL_ENTRY();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    uint32_t rank, ranks;
    asm("mov.u32 %0, %cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %cluster_nctarank;" : "=r"(ranks));
    const int unit = blockIdx.x / ranks, kh = unit % p.Hkv, b = unit / p.Hkv;
    int32_t* const out = p.out + (size_t)unit * p.K;
    const int step = (int)ranks * kRows, start = (int)rank * kRows + warp * 32;
    // A lane's block of the warp's 32: its first page.  Asked for beside the lengths, as far as the table has columns; a block behind the context is not used.
    auto page_of = [&](int base) {
        const long long col = (long long)(base + lane) << (p.shift - 4);
        return col < p.max_pages ? __ldg(p.table + (size_t)b * p.max_pages + col) : -1;
    };
    int page_next = page_of(start);
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
        if (rank == 0)
            for (int k = tid; k < p.K; k += kThreads) out[k] = k < nb ? k : -1;
        if (error && tid == 0 && kh == 0 && rank == 0) atomicCAS(p.status, 0u, (uint32_t)error);
        return;
    }
    if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int nq = n * p.G;
    auto query = [&](int i) { return p.q + ((size_t)(row0 + i / p.G) * p.Hq + kh * p.G + i % p.G) * D; };
    // 32 blocks' summaries: rows gid and gid + 8 of two groups of 16; lane l keeps block l's scale
    uint32_t a[2][2][W];
    float scale = 0.f;
    bool good = true;
    auto load_rows = [&](int base) {
        int page = page_next;
        good = base + lane >= nb || (page >= 0 && page < p.num_pages);
        if (!good || base + lane >= nb) page = 0;
        if (base + step < nb) page_next = page_of(base + step);
        scale = good ? __ldg(p.scale + (size_t)page * p.Hkv + kh) : 0.f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int pg = __shfl_sync(CB_FULL, page, g * 8 + gid);
            const uint4* src = reinterpret_cast<const uint4*>(p.mean + ((size_t)pg * p.Hkv + kh) * D + tig * 16);
#pragma unroll
            for (int c = 0; c < W / 4; ++c) {
                const uint4 v = __ldg(src + c * 4);
                uint32_t* w = &a[g >> 1][g & 1][c * 4];
                w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            }
        }
    };
    if (start < nb) load_rows(start);                         // on their way while the queries are made ready
    // largest magnitude of the queries, as bits of bf16
    uint32_t top = 0;
    for (int k = tid; k < nq * (D / 8); k += kThreads) {
        const uint4 v = *reinterpret_cast<const uint4*>(query(k / (D / 8)) + k % (D / 8) * 8);
        top = __vmaxu2(top, __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)));
    }
    top = max(top & 0xFFFFu, top >> 16);
    top = __reduce_max_sync(CB_FULL, top);
    if (lane == 0) s_warp[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = max(top, s_warp[w]);
    const float r = __fdiv_rn(127.f, fmaxf(__uint_as_float(top << 16), 1e-30f));
    // Query i's 16-byte piece c lies at piece c ^ (i & 1) * W / 8 * 4 of its row, so that eight lanes that read two rows meet no bank twice.
    auto piece = [&](int i, int c) { return s_q + i * D + ((D == 128 ? c ^ ((i & 1) << 2) : c) << 4); };
    auto make_queries = [&](int q0, int nt) {
        const int padded = (nt + 7) & ~7;                     // the last tile of eight is filled up with its first query
        for (int k = tid; k < padded * (D / 16); k += kThreads) {
            const int i = k / (D / 16), c = k % (D / 16);
            const uint4* src = reinterpret_cast<const uint4*>(query(q0 + (i < nt ? i : 0)) + c * 16);
            uint32_t o[4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 v = src[h];
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // adding 1.5 * 2^23 rounds to a whole number and leaves it in the low bits (a conversion is a quarter as fast)
                    auto whole = [&](uint32_t bits) { return __float_as_uint(__fadd_rn(__fmul_rn(__uint_as_float(bits), r), 12582912.f)); };
                    const uint32_t x0 = whole(w[2 * e] << 16), x1 = whole(w[2 * e] & 0xFFFF0000u), x2 = whole(w[2 * e + 1] << 16), x3 = whole(w[2 * e + 1] & 0xFFFF0000u);
                    o[2 * h + e] = __byte_perm(__byte_perm(x0, x1, 0x0040), __byte_perm(x2, x3, 0x0040), 0x5410);
                }
            }
            *reinterpret_cast<uint4*>(piece(i, c)) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    };
    auto load_tile = [&](int i0, uint32_t* w) {
#pragma unroll
        for (int c = 0; c < W / 4; ++c) {
            const uint4 v = *reinterpret_cast<const uint4*>(piece(i0 + gid, tig + 4 * c));
            w[4 * c] = v.x; w[4 * c + 1] = v.y; w[4 * c + 2] = v.z; w[4 * c + 3] = v.w;
        }
    };
    int best[2][2];
    auto score_tile = [&](const uint32_t* w) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            int c[4] = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < W / 2; ++s) mma_s8(c, a[g][0][s], a[g][1][s], a[g][0][s + W / 2], a[g][1][s + W / 2], w[s], w[s + W / 2]);
            best[g][0] = max(best[g][0], max(c[0], c[1]));
            best[g][1] = max(best[g][1], max(c[2], c[3]));
        }
    };
    // lane l: the largest product of block l of the warp's 32
    auto row_best = [&] {
        int mine = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            int v = best[g >> 1][g & 1];
            v = max(v, __shfl_xor_sync(CB_FULL, v, 1));
            v = max(v, __shfl_xor_sync(CB_FULL, v, 2));
            v = __shfl_sync(CB_FULL, v, (lane & 7) * 4);
            if ((lane >> 3) == g) mine = v;
        }
        return mine;
    };
    uint32_t key0 = 0;                                        // the first CTA's keys, which all of a cluster write to
    if (ranks > 1) {
        asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(key0) : "r"((uint32_t)__cvta_generic_to_shared(s_key)));
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    for (int q0 = 0; q0 < nq; q0 += NT ? NT * 8 : p.tile) {
        const int nt = min(NT ? NT * 8 : p.tile, nq - q0);
        if (q0 > 0) __syncthreads();
        make_queries(q0, nt);
        __syncthreads();
        uint32_t w[NT ? NT : 1][W];
        if (NT) {
#pragma unroll
            for (int k = 0; k < NT; ++k)
                if (k * 8 < nt) load_tile(k * 8, w[k]);
        }
        for (int base = start; base < nb; base += step) {
            if (q0 > 0 && base == start) page_next = page_of(start);
            if (base != start || q0 > 0) load_rows(base);
            best[0][0] = best[0][1] = best[1][0] = best[1][1] = INT32_MIN;
            if (NT) {
#pragma unroll
                for (int k = 0; k < NT; ++k)
                    if (k * 8 < nt) score_tile(w[k]);
            } else {
                for (int i = 0; i < nt; i += 8) {
                    load_tile(i, w[0]);
                    score_tile(w[0]);
                }
            }
            int m = row_best();
            const int j = base + lane;
            if (j < nb) {
                if (q0 > 0) m = max(m, (int)s_key[j]);
                if (q0 + nt < nq) s_key[j] = (uint32_t)m;     // (of a later tile's queries more)
                else {
                    const uint32_t key = score_key(m, scale);
                    if (ranks > 1) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(key0 + 4u * (uint32_t)j), "r"(key) : "memory");
                    else s_key[j] = key;
                    if (!good) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
                }
            }
            __syncwarp();
        }
    }
    if (ranks > 1) {
        cluster_sync();
        if (rank != 0) return;
    }
    __syncthreads();
    const int lo = p.n_first, hi = nb - p.n_last;
    uint32_t left = (uint32_t)(p.K - p.n_first - p.n_last);
    if (nb <= 2 * kThreads) {
        // Two keys a thread, in registers.  The want-th largest is found bit by bit below the highest one in which keys differ, a count by barrier each, and
        // early where a bound has just as many keys above it as are wanted.  (No candidate's key is 0.)
        const bool c0 = tid >= lo && tid < hi, c1 = tid + kThreads >= lo && tid + kThreads < hi;
        const uint32_t k0 = c0 ? s_key[tid] : 0u, k1 = c1 ? s_key[tid + kThreads] : 0u;
        const bool second = nb > kThreads;
        const uint32_t least = __reduce_min_sync(CB_FULL, min(c0 ? k0 : 0xFFFFFFFFu, c1 ? k1 : 0xFFFFFFFFu)), most = __reduce_max_sync(CB_FULL, max(k0, k1));
        if (lane == 0) { s_warp[warp] = least; s_eq[warp] = most; }
        __syncthreads();
        uint32_t low = least, high = most;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) { low = min(low, s_warp[w]); high = max(high, s_eq[w]); }
        uint32_t bound = 0xFFFFFFFFu, equals = 0;             // chosen: keys above the bound and the first of its equals
        bool from = false;                                    // or all keys from it on
        if (left > 0) {
            auto count = [&](uint32_t x) { return (uint32_t)(__syncthreads_count(k0 >= x) + (second ? __syncthreads_count(k1 >= x) : 0)); };
            const int differ = 31 - __clz(low ^ high);        // -1: all are equal
            bound = differ < 31 ? high & ~((2u << differ) - 1u) : 0u;
            if (differ < 0) bound = high;
            for (int bit = differ; bit >= 0 && !from; --bit) {
                const uint32_t x = bound | (1u << bit), c = count(x);
                if (c >= left) bound = x;
                from = c == left;
            }
            if (!from) equals = left - (bound == 0xFFFFFFFFu ? 0u : count(bound + 1u));
        }
        const bool any = left > 0;
        auto over = [&](int j, bool cand, uint32_t key) { return j < nb && (!cand || (any && (from ? key >= bound : key > bound))); };
        auto equal = [&](bool cand, uint32_t key) { return cand && any && !from && key == bound; };
        const uint32_t o0 = __ballot_sync(CB_FULL, over(tid, c0, k0)), e0 = __ballot_sync(CB_FULL, equal(c0, k0));
        const uint32_t o1 = __ballot_sync(CB_FULL, over(tid + kThreads, c1, k1)), e1 = __ballot_sync(CB_FULL, equal(c1, k1));
        if (lane == 0) { s_hist[warp] = __popc(o0) | __popc(e0) << 16; s_hist[kWarps + warp] = __popc(o1) | __popc(e1) << 16; }
        __syncthreads();
        uint32_t sum = lane < 2 * kWarps ? s_hist[lane] : 0u;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(CB_FULL, sum, o); if (lane >= o) sum += y; }
        const uint32_t b0 = warp == 0 ? 0u : __shfl_sync(CB_FULL, sum, (warp + 31) & 31), b1 = __shfl_sync(CB_FULL, sum, kWarps + warp - 1);
        const uint32_t under = (1u << lane) - 1u;
        auto put = [&](int j, uint32_t before, uint32_t o, uint32_t e) {
            const uint32_t g = (before & 0xFFFFu) + __popc(o & under), q = (before >> 16) + __popc(e & under);
            if ((o >> lane & 1u) || ((e >> lane & 1u) && q < equals)) out[g + min(q, equals)] = j;
        };
        put(tid, b0, o0, e0);
        put(tid + kThreads, b1, o1, e1);
        return;
    }
    // More keys: eight bits at a time below the highest bit in which keys differ, by counts of the digits, and early where a digit's keys are all wanted.
    uint32_t least = 0xFFFFFFFFu, most = 0;
    const bool any = left > 0;
    for (int j = lo + tid; j < hi; j += kThreads) { const uint32_t k = s_key[j]; least = min(least, k); most = max(most, k); }
    least = __reduce_min_sync(CB_FULL, least); most = __reduce_max_sync(CB_FULL, most);
    if (lane == 0) { s_warp[warp] = least; s_eq[warp] = most; }
    if (tid < 256) s_hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) { least = min(least, s_warp[w]); most = max(most, s_eq[w]); }
    uint32_t prefix = 0;                                      // of key - least
    bool from = false;                                        // all keys from the prefix on; else those above it, and `left` of its equals
    if (any)
        for (int bits = max(24 - __clz(most - least), 0), above = 32; ; above = bits, bits = max(bits - 8, 0)) {
            const int width = min(above, 32) - bits;          // (the first digit has what is above it zero)
            for (int j = lo + tid; j < hi; j += kThreads) {
                const uint32_t k = s_key[j] - least;
                if (above >= 32 || (k >> above) == (prefix >> above)) atomicAdd(&s_hist[(k >> bits) & (width >= 8 ? 255u : (1u << width) - 1u)], 1u);
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
                        if (before < left && left <= before + c[e]) { s_pick[0] = prefix | ((uint32_t)(255 - (lane * 8 + e)) << bits); s_pick[1] = left - before; s_pick[2] = c[e]; }
                        before += c[e];
                    }
                }
            }
            __syncthreads();
            prefix = s_pick[0]; left = s_pick[1];
            from = s_pick[2] == left;
            if (from || bits == 0) break;
            if (tid < 256) s_hist[tid] = 0;
            __syncthreads();
        }
    auto over = [&](int j) { return j < lo || j >= hi || (any && (from ? s_key[j] - least >= prefix : s_key[j] - least > prefix)); };
    auto equal = [&](int j) { return j >= lo && j < hi && any && !from && s_key[j] - least == prefix; };
    // In order: a run of blocks per thread, where its chosen ones go by the sums before it.
    const int run = (nb + kThreads - 1) / kThreads, j0 = min(tid * run, nb), j1 = min(j0 + run, nb);
    uint32_t gt = 0, eq = 0;
    for (int j = j0; j < j1; ++j) { gt += over(j); eq += equal(j); }
    uint32_t gs = gt, es = eq;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(CB_FULL, gs, o), z = __shfl_up_sync(CB_FULL, es, o);
        if (lane >= o) { gs += y; es += z; }
    }
    __syncthreads();
    if (lane == 31) { s_warp[warp] = gs; s_eq[warp] = es; }
    __syncthreads();
    gs -= gt; es -= eq;
    for (int w = 0; w < warp; ++w) { gs += s_warp[w]; es += s_eq[w]; }
    for (int j = j0; j < j1; ++j) {
        const bool o = over(j), e = equal(j);
        if (o || (e && es < left)) out[gs + min(es, left)] = j;
        gs += o; es += e;
    }
}

std::mutex g_mutex;
size_t g_smem[6][64];

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
    p.key_words = (blocks + 3) & ~3;
    // Queries of 8 or 16 rows and heads stay in registers; more go through shared memory, 512 at a time.
    const long long votes = (long long)(a->q_start ? p.max_chunk : p.T) * p.G;
    const int nt = votes <= 8 ? 1 : (votes <= 16 ? 2 : 0);
    p.tile = nt ? nt * 8 : (int)std::min<long long>(kSelQueries, (votes + 7) & ~7ll);
    const size_t smem = (size_t)p.key_words * 4 + (size_t)p.tile * c.head_dim;
    // With few units a cluster shares each one's blocks, as many CTAs as there are SMs for and 32 blocks a warp keep busy.
    int ctas = 1;
    while (ctas < 8 && (long long)p.B * p.Hkv * ctas * 2 <= ctx->num_sms && blocks > ctas * sel_threads(nt) / 2) ctas *= 2;
    const auto launch = [&](auto kernel, int which) -> cb_status {
        {
            std::lock_guard<std::mutex> lock(g_mutex);
            size_t fresh = 0;
            CB_CUDA(cb_allow_smem(kernel, smem, ctx->device >= 0 && ctx->device < 64 ? &g_smem[which][ctx->device] : &fresh));
        }
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((long long)p.B * p.Hkv * ctas)); cfg.blockDim = dim3(sel_threads(nt)); cfg.dynamicSmemBytes = smem; cfg.stream = (cudaStream_t)stream;
        cudaLaunchAttribute at[2];
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
        at[1].id = cudaLaunchAttributeClusterDimension;
        at[1].val.clusterDim.x = (unsigned)ctas; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
        cfg.attrs = at; cfg.numAttrs = 2;
        CB_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
        cb_count_launch(1);
        return CB_OK;
    };
    if (c.head_dim == 128) return nt == 1 ? launch(cb_block_select_kernel<128, 1>, 0) : (nt == 2 ? launch(cb_block_select_kernel<128, 2>, 1) : launch(cb_block_select_kernel<128, 0>, 2));
    return nt == 1 ? launch(cb_block_select_kernel<64, 1>, 3) : (nt == 2 ? launch(cb_block_select_kernel<64, 2>, 4) : launch(cb_block_select_kernel<64, 0>, 5));
}
