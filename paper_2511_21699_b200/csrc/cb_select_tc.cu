// Selection of blocks by many queries (trees, chunks), on the 5th-generation tensor cores.
//
// A CTA, or a cluster that deals a unit's tiles of 128 blocks among its CTAs, per (sequence, kv head).  Scores are products of bytes, tcgen05 kind::i8: 128 blocks by
// up to 256 queries, in 32-bit whole numbers, into one of two halves of tensor memory.  What is wanted of them is the largest of each block's row, and a row lies in
// one lane of tensor memory, so that a thread finds it alone: eight warps take a half's 256 columns, 128 each, while the other half is being filled.
// Queries and summaries are put into shared memory 512 at a time, 128 bytes a row with the 128-byte swizzle (half of a row unused with 64 dims).
//
// Measured: 16 trees of 64 nodes, 64 query heads over 8, contexts of 16 k to 32 k in blocks of 64: 16 us (209 with __dp4a by a thread per block, 25.6 with m16n8k32 products).  A
// unit's phases follow one another: lengths and pages 3.5 k cycles, the queries' largest magnitude 5 k (17 MB from memory over all units), whole numbers 4 k, eight jobs 7 k, search 1.5 k.
#include <mutex>

#include "cb_select.cuh"
#include "cb_tc_dev.cuh"

namespace {

constexpr int kManyWorkers = 512, kManyThreads = kManyWorkers + 32;   // and a warp that issues the products
constexpr int kManyRows = 512;                                // blocks, and queries, in shared memory at a time
// Shared memory: queries, summaries, barriers and flags, pages, then the keys.
constexpr uint32_t kOffRows = kManyRows * 128, kOffBar = 2 * kManyRows * 128, kOffMisc = kOffBar + 64, kOffScratch = kOffMisc + 64,
                   kScratchWords = cb_pick_words<kManyThreads>, kOffPage = kOffScratch + kScratchWords * 4, kOffKey = kOffPage + kManyRows * 4;
static_assert(kOffKey % 16 == 0, "keys in pieces of 16 bytes");

// 128 blocks x N queries of D bytes each: whole numbers of 32 bits, signed bytes on both sides.
__host__ __device__ constexpr uint32_t idesc_i8(int n) { return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24); }
__device__ __forceinline__ void mma_i8(uint32_t d, uint32_t alo, uint32_t blo, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %4, p;\n\t}"
        ::"r"(d), "r"(alo), "r"(blo), "r"(kDescHi), "r"(idesc), "r"((uint32_t)add) : "memory");
}

template <int D>
__global__ void __launch_bounds__(kManyThreads, 1) cb_select_many_kernel(const CbSelectParams p) {
    constexpr int L = D / 16;                                 // 16-byte pieces of a row
    extern __shared__ __align__(1024) uint8_t select_smem[];
    uint8_t *const s_q = select_smem, *const s_rows = select_smem + kOffRows;
    uint32_t *const s_scratch = reinterpret_cast<uint32_t*>(select_smem + kOffScratch), *const s_key = reinterpret_cast<uint32_t*>(select_smem + kOffKey);
    int* const s_page = reinterpret_cast<int*>(select_smem + kOffPage);
    uint32_t* const s_tmem = reinterpret_cast<uint32_t*>(select_smem + kOffMisc);
    volatile int* const s_abort = reinterpret_cast<volatile int*>(select_smem + kOffMisc + 4);
    const uint32_t bars = smem_u32(select_smem + kOffBar);
    auto bar_full = [&](int h) { return bars + 8u * h; };     // half h of tensor memory holds scores
    auto bar_free = [&](int h) { return bars + 8u * (2 + h); };   // eight warps have read it
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (smem_u32(select_smem) & 1023u) {                      // the swizzled tiles need it; every thread sees the same address
        if (tid == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_UNSUPPORTED);
        return;
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        if (lane == 0) {
            for (int h = 0; h < 2; ++h) { mbar_init(bar_full(h), 1); mbar_init(bar_free(h), 8); }
            *s_abort = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();                                          // the tensor memory is held before the next kernel's blocks may come
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    CB_PDL_ENTRY();
    uint32_t rank, ranks;
    asm("mov.u32 %0, %cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %cluster_nctarank;" : "=r"(ranks));
    const int unit = blockIdx.x / ranks;
    // The CTA's i-th block: tiles of 128 are dealt to the cluster's CTAs in turn.
    auto block_of = [&](int i) { return ((i >> 7) * (int)ranks + (int)rank) * 128 + (i & 127); };
    auto page_of = [&](int j) {
        const long long col = (long long)j << (p.shift - 4);
        return col < p.max_pages ? p.table[(size_t)(unit / p.Hkv) * p.max_pages + col] : -1;
    };
    int page = page_of(block_of(tid));                        // of the first 512, beside the lengths
    const CbSelectUnit u = cb_select_unit(p, unit, rank == 0, tid, kManyThreads);
    const int nb = u.nb, nq = u.n * p.G;
    const bool worker = warp < kManyWorkers / 32;
    bool ok = true;
    if (nb > 0) {
        const int tiles = (nb + 127) / 128, own = (int)rank < tiles ? ((tiles - 1 - (int)rank) / (int)ranks + 1) * 128 : 0;   // places of this CTA's blocks
        auto at_swizzled = [&](uint8_t* base, int row, int c) { return base + row * 128 + ((c ^ (row & 7)) << 4); };
        // 512 blocks' summaries into shared memory; thread i keeps block i's page there
        auto load_rows = [&](int i0) {
            const int j = block_of(i0 + tid);
            if (i0 > 0) page = i0 + tid < own ? page_of(j) : -1;
            const bool there = i0 + tid < own && j < nb;
            const bool good = page >= 0 && page < p.num_pages;
            if (there && !good) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
            s_page[tid] = there && good ? page : -1;
            __syncwarp();
            const int rows = min(32, own - i0 - warp * 32);   // a warp copies its lanes' blocks
            for (int k = lane; k < rows * L; k += 32) {
                const int row = warp * 32 + k / L, c = k % L, pg = max(s_page[row], 0);
                const int8_t* src = p.mean + ((size_t)pg * p.Hkv + u.kh) * D + c * 16;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(at_swizzled(s_rows, row, c))), "l"(src) : "memory");
            }
        };
        if (worker && own > 0) load_rows(0);
        // 512 queries, eight 16-byte pieces of a thread under way at a time: to find their largest magnitude, and again (from L2) to make whole numbers of them.
        constexpr int V = kManyRows * (D / 8) / kManyWorkers, STEP = V < 8 ? V : 8;
        auto queries = [&](int q0, auto&& use) {
            const int n = min(kManyRows, nq - q0), padded = min((n + 31) & ~31, kManyRows);   // (filled up with the first one)
#pragma unroll 1
            for (int k0 = 0; k0 < V; k0 += STEP) {
                if (k0 * kManyWorkers >= padded * (D / 8)) break;
                uint4 v[STEP];
#pragma unroll
                for (int k = 0; k < STEP; ++k) {
                    const int x = (k0 + k) * kManyWorkers + tid, i = x / (D / 8);
                    v[k] = *reinterpret_cast<const uint4*>(cb_select_query<D>(p, u, q0 + (i < n ? i : 0)) + x % (D / 8) * 8);
                }
#pragma unroll
                for (int k = 0; k < STEP; ++k) use((k0 + k) * kManyWorkers + tid, v[k]);
            }
        };
        uint32_t top = 0;
        if (worker)
            for (int q0 = 0; q0 < nq; q0 += kManyRows) queries(q0, [&](int, const uint4& v) { top = cb_max_bits(top, v); });
        top = __reduce_max_sync(CB_FULL, max(top & 0xFFFFu, top >> 16));
        if (lane == 0) s_scratch[warp] = top;
        for (int j = tid; j < p.key_words; j += kManyThreads) s_key[j] = 0x80000000u;
        __syncthreads();
        if (ranks > 1) cb_cluster_arrive();                   // (from here on its keys may be written by the others)
#pragma unroll
        for (int w = 0; w < kManyThreads / 32; ++w) top = max(top, s_scratch[w]);
        const float r = cb_whole_factor(top);
        // Jobs: a tile of 128 blocks by up to 256 queries each, counted over the whole launch; job e fills half e & 1, whose eight warps are those with
        // (warp >> 3) == (e & 1).  A warp's quarter of the lanes is fixed; of the two that share it, one takes the first 128 columns, one the others.
        uint32_t jobs = 0;
        const int mine = (warp >> 3) & 1, columns = (warp >> 2) & 1, quarter = warp & 3;
        bool stop = false;                                    // a wait ran out: known to all threads at once
        for (int q0 = 0; q0 < nq && !stop; q0 += kManyRows) {
            const int n = min(kManyRows, nq - q0), padded = (n + 31) & ~31, halves = (padded + 255) / 256;
            if (q0 > 0) __syncthreads();                      // the products of the queries before have been read
            if (worker)
                queries(q0, [&](int x, const uint4& v) {
                    const int c = x % (D / 8);
                    *reinterpret_cast<uint2*>(at_swizzled(s_q, x / (D / 8), c >> 1) + (c & 1) * 8) = cb_whole8(v, r);
                });
            for (int i0 = 0; i0 < own && !stop; i0 += kManyRows) {
                if (i0 > 0 || (q0 > 0 && own > kManyRows)) {
                    __syncthreads();
                    if (i0 == 0) page = page_of(block_of(tid));
                    if (worker) load_rows(i0);
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                stop = __syncthreads_or(!ok);
                if (stop) break;
                const int mt = min(kManyRows, own - i0) / 128, count = mt * halves;
                if (!worker) {
                    if (elect_one())
                        for (int e = 0; e < count; ++e) {
                            const uint32_t job = jobs + e;
                            const int h = (int)(job & 1u), m = e / halves, q = e - m * halves, cols = min(256, padded - q * 256);
                            if (job >= 2 && !(ok = mbar_wait(bar_free(h), (job / 2 - 1) & 1, s_abort, p.status))) break;
                            tc_fence_after();
                            const uint32_t alo = desc_lo(smem_u32(s_rows) + m * 128 * 128, 16), blo = desc_lo(smem_u32(s_q) + q * 256 * 128, 16);
#pragma unroll
                            for (int k = 0; k < D / 32; ++k) mma_i8(tmem + h * 256, alo + 2 * k, blo + 2 * k, idesc_i8(cols), k > 0);
                            tc_commit(bar_full(h));
                        }
                    __syncwarp();
                } else {
                    for (int e = (int)((mine - jobs) & 1u); e < count; e += 2) {
                        const uint32_t job = jobs + e;
                        const int m = e / halves, q = e - m * halves, cols = min(256, padded - q * 256);
                        if (!(ok = __all_sync(CB_FULL, mbar_wait(bar_full(mine), (job / 2) & 1, s_abort, p.status)))) break;   // (all lanes go on, or none)
                        tc_fence_after();
                        int best = INT32_MIN;
                        // (64 columns under way at once, what lies behind the last query's 32 not looked at)
                        for (int c = columns * 128; c < min(cols, columns * 128 + 128); c += 64) {
                            uint32_t x[32], y[32];
                            const uint32_t at = tmem + mine * 256 + c + ((uint32_t)(quarter * 32) << 16);
                            CB_TMEM_LD32(x, 0, at);
                            if (c + 32 < cols) CB_TMEM_LD32(y, 0, at + 32);
                            CB_TMEM_WAIT_LD32(x);
#pragma unroll
                            for (int k = 0; k < 32; k += 2) best = max(best, max((int)x[k], (int)x[k + 1]));
                            if (c + 32 < cols) {
                                CB_TMEM_WAIT_LD32(y);
#pragma unroll
                                for (int k = 0; k < 32; k += 2) best = max(best, max((int)y[k], (int)y[k + 1]));
                            }
                        }
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar_free(mine));
                        const int j = block_of(i0 + m * 128 + quarter * 32 + lane);
                        if (j < nb && columns * 128 < cols) atomicMax(reinterpret_cast<int*>(s_key) + j, best);
                    }
                    __syncwarp();
                }
                jobs += (uint32_t)count;
            }
        }
        // the keys, in the cluster's first CTA
        __syncthreads();
        for (int k = tid; k < (int)kScratchWords; k += kManyThreads) s_scratch[k] = 0u;
        const uint32_t key0 = ranks > 1 ? cb_cluster_first(s_key) : 0u;
        if (ranks > 1) cb_cluster_wait();
        for (int i = tid; i < own; i += kManyThreads) {
            const int j = block_of(i);
            if (j >= nb) break;
            const int pg = own <= kManyRows ? s_page[i] : page_of(j);
            const uint32_t key = cb_score_key((int)s_key[j], pg >= 0 && pg < p.num_pages ? p.scale[(size_t)pg * p.Hkv + u.kh] : 0.f);
            if (ranks > 1) cb_cluster_store(key0 + 4u * (uint32_t)j, key);
            else s_key[j] = key;
        }
        __syncwarp();
        if (ranks > 1) { cb_cluster_arrive(); cb_cluster_wait(); }
        __syncthreads();
        if (rank == 0) cb_pick<kManyThreads>(p, nb, s_key, s_scratch, p.out + (size_t)unit * p.K);
    }
    if (*s_abort)                                             // products that are still under way
        for (int k = 0; k < 64; ++k) __nanosleep(1000);
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

std::mutex g_mutex;
size_t g_smem[2][64];

}  // namespace

cb_status cb_select_launch_many(const cb_ctx* ctx, const CbSelectParams& p, int ctas, cudaStream_t st) {
    const size_t smem = kOffKey + (size_t)p.key_words * 4;
    if (smem > 227 * 1024) return CB_ERR_UNSUPPORTED;
    const auto launch = [&](auto kernel, int which) -> cb_status {
        {
            std::lock_guard<std::mutex> lock(g_mutex);
            size_t fresh = 0;
            CB_CUDA(cb_allow_smem(kernel, smem, ctx->device >= 0 && ctx->device < 64 ? &g_smem[which][ctx->device] : &fresh));
        }
        CB_CUDA(cb_launch_clusters(kernel, (unsigned)((long long)p.B * p.Hkv * ctas), (unsigned)ctas, kManyThreads, smem, st, p));
        cb_count_launch(1);
        return CB_OK;
    };
    return ctx->cfg.head_dim == 128 ? launch(cb_select_many_kernel<128>, 1) : launch(cb_select_many_kernel<64>, 0);
}
