// Block tables kept on the GPU: pages to the sequences that grow and back from those that shrink, and where a packed batch's rows go.
//
// cb_pages_assign.  With back(b) and need(b) the pages that sequence b gives back and asks for, everything follows from their sums over the batch, which
// every CTA takes for itself.  The j-th page handed out is the j-th one given back or, behind those, the stack's from its top; it goes to the sequence whose
// sum of needs passes j.  So all moves are independent: a thread finds both sequences of a move by two searches in shared memory.  Pages given back
// that nobody takes are pushed above the old top, pages taken from the stack lie below it, rows that are read belong to sequences that shrink and rows
// that are written to such that grow: no move touches what another one reads.  held and n_free, which all CTAs read, are written by the one that counted itself
// last behind that.  How many moves there are is known on the device only: a table of up to 16,384 entries gets one CTA, a larger one as many
// as it has 2,048 entries, one an SM at most.  (A step of 32 sequences, one CTA against that many: 3.8 and 4.0 us with 16,384 entries, 3.8 and 3.9 with 32,768; calls that move a
// quarter of the table: 6.0 and 3.9, 8.9 and 4.1, with 65,536 entries 15 and 4.0.  With a CTA for 8,192 entries 5.0, for 512 as for 2,048.)  Round trips bound it: 3.5 us a call for
// 32 sequences of which half take a page, 5.5 for 512 sequences that take or give back 133,000 (a cluster of eight CTAs: 6.6 and 24).
//
// cb_slot_map.  A thread per row: the sequence by a search in the block's copy of q_start, then its length and page.  The launch bounds it: 3.1 us a call for 32 rows and
// for 66,000.
#include <algorithm>

#include "cb_scan.cuh"

namespace {

constexpr int kPageThreads = 1024;

__global__ void __launch_bounds__(kPageThreads) cb_pages_assign_kernel(int B, int P, int max_pages, int num_pages, const int32_t* want_len, int32_t* table,
                                                                       int32_t* held, int32_t* stack, int32_t* n_free, uint32_t* ticket, uint32_t* status) {
    extern __shared__ uint32_t s_sums[];                      // [2][B]: needs, pages given back
    __shared__ uint32_t s_scratch[2 * kPageThreads / 32];
    __shared__ int s_last;
    uint32_t *const s_need = s_sums, *const s_back = s_sums + B;
    CB_PDL_ENTRY();
    const int tid = threadIdx.x;
    const int free0 = n_free[0];
    int error = free0 < 0 || free0 > num_pages ? CB_ERR_INVALID_ARG : 0;
    const bool stack_ok = error == 0;
    // pages that the sequence is to hold; -1: it is left alone
    auto pages_of = [&](int w) { return w / P + (w % P != 0); };
    auto target = [&](int b, int h, int* why) {
        const int w = want_len[b];
        if (w < 0 || h < 0 || h > max_pages) { *why = CB_ERR_INVALID_ARG; return -1; }
        const int t = pages_of(w);
        if (t > max_pages) { *why = CB_ERR_KV_FULL; return -1; }
        return t;
    };
    cb_block_sums<kPageThreads, 2>(B, s_sums, s_scratch, [&](int b, uint32_t* c) {
        const int h = held[b];
        const int t = target(b, h, &error);
        if (t >= 0) { c[0] = min((uint32_t)max(t - h, 0), CB_SUM_CAP); c[1] = min((uint32_t)max(h - t, 0), CB_SUM_CAP); }
    });
    // (the barrier behind the sums lies behind every thread's reads of held and n_free)
    const bool many = gridDim.x > 1;
    if (many && tid == 0) {
        __threadfence();
        s_last = atomicAdd(ticket, 1u) == gridDim.x - 1u;
    }
    const uint32_t gone = s_back[B - 1], there = (uint32_t)free0 + gone;
    const bool ok = stack_ok && there <= (uint32_t)num_pages;
    // needs that are met: up to the largest sum that does not exceed what is there
    const int met = ok ? cb_upper(s_need, B, there) : 0;
    const uint32_t taken = met > 0 ? s_need[met - 1] : 0u;
    if (ok) {
        auto given_back = [&](uint32_t i) {                   // the i-th page given back
            const int b = cb_upper(s_back, B, i);
            return table[(size_t)b * max_pages + pages_of(want_len[b]) + (int)(i - (b > 0 ? s_back[b - 1] : 0u))];
        };
        const uint32_t step = gridDim.x * kPageThreads;
        for (uint32_t j = blockIdx.x * kPageThreads + tid; j < taken; j += step) {
            const int b = cb_upper(s_need, B, j);
            const int page = j < gone ? given_back(j) : stack[there - 1u - j];
            table[(size_t)b * max_pages + pages_of(want_len[b]) - (int)(s_need[b] - j)] = page;
        }
        for (uint32_t i = taken + blockIdx.x * kPageThreads + tid; i < gone; i += step) stack[there - 1u - i] = given_back(i);
    }
    if (many) {
        __syncthreads();
        if (!s_last) return;
        if (tid == 0) *ticket = 0u;
    }
    if (ok)
        for (int b = tid; b < B; b += kPageThreads) {
            int why = 0;
            const int h = held[b], t = target(b, h, &why);
            if (t > h && b >= met) error = CB_ERR_KV_FULL;
            else if (t >= 0 && t != h) held[b] = t;
        }
    if (!ok) error = CB_ERR_INVALID_ARG;
    else if (tid == 0) n_free[0] = (int)(there - taken);
    if (error) atomicCAS(status, 0u, (uint32_t)error);
}

constexpr int kSlotThreads = 256, kSlotSeqs = 2048;           // sequences whose starts a block keeps

__global__ void __launch_bounds__(kSlotThreads) cb_slot_map_kernel(int B, int P, int max_pages, int num_pages, int n_rows, const int32_t* q_start,
                                                                   const int32_t* ctx_len, const int32_t* table, int64_t* slots,
                                                                   int32_t* positions, int32_t* seqs, uint32_t* status) {
    __shared__ int32_t s_start[kSlotSeqs];
    CB_PDL_ENTRY();
    const int tid = threadIdx.x;
    auto wrong = [&](int q0, int q1, int ctx) {
        if (q0 == q1) return 0;
        if (q0 < 0 || q1 < q0 || q1 > n_rows || ctx < 0) return (int)CB_ERR_INVALID_ARG;
        return (long long)ctx + (q1 - q0) > (long long)max_pages * P || ctx > 0x7FFFFFFF - (q1 - q0) ? (int)CB_ERR_KV_FULL : 0;
    };
    if (blockIdx.x == gridDim.x - 1)                          // behind the rows' blocks one that looks the sequences over
        for (int b = tid; b < B; b += kSlotThreads) {
            const int e = wrong(q_start[b], q_start[b + 1], ctx_len[b]);
            if (e) atomicCAS(status, 0u, (uint32_t)e);
        }
    const bool kept = B <= kSlotSeqs;
    if (kept) {
        for (int b = tid; b < B; b += kSlotThreads) s_start[b] = q_start[b];
        __syncthreads();
    }
    const long long r64 = (long long)blockIdx.x * kSlotThreads + tid;
    if (r64 >= n_rows) return;
    const int r = (int)r64;
    int lo = 0, n = B;                                        // the last sequence with q_start <= r
    const int32_t* const start = kept ? s_start : q_start;
    while (n > 0) {
        const int h = n >> 1;
        if (start[lo + h] > r) n = h;
        else { lo += h + 1; n -= h + 1; }
    }
    int64_t slot = -1;
    int pos = -1, b = lo - 1;
    if (b >= 0) {
        const int q0 = start[b], q1 = q_start[b + 1], ctx = ctx_len[b];
        if (r >= q1 || wrong(q0, q1, ctx)) b = -1;
        else {
            pos = ctx + (r - q0);
            const int page = table[(size_t)b * max_pages + pos / P];
            if (page >= 0 && page < num_pages) slot = (int64_t)page * P + pos % P;
            else atomicCAS(status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
        }
    }
    slots[r] = slot;
    positions[r] = pos;
    seqs[r] = b;
}

}  // namespace

extern "C" cb_status cb_pages_assign(cb_ctx* ctx, const int32_t* want_len, int32_t* block_table, int32_t max_pages, int32_t* held, int32_t* free_pages,
                                     int32_t num_pages, int32_t* n_free, void* stream) {
    CB_CHECK_ARG(ctx && want_len && block_table && held && free_pages && n_free && max_pages >= 1 && num_pages >= 1);
    const cb_config& c = ctx->cfg;
    if (c.batch > CB_MAX_ASSIGN || num_pages >= (int)CB_SUM_CAP) return CB_ERR_UNSUPPORTED;   // (a capped sum of needs exceeds all there can be)
    const size_t smem = (size_t)c.batch * 8;
    if (smem > 40 * 1024) CB_CUDA(cudaFuncSetAttribute(cb_pages_assign_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, CB_MAX_ASSIGN * 8));
    const long long entries = (long long)c.batch * max_pages;
    const unsigned ctas = entries <= 16384 ? 1u : (unsigned)std::min<long long>(entries / 2048, ctx->num_sms);
    CB_CUDA(cb_launch_pdl(cb_pages_assign_kernel, dim3(ctas), dim3(kPageThreads), smem, (cudaStream_t)stream, (int)c.batch, (int)c.page_size, (int)max_pages,
                          (int)num_pages, want_len, block_table, held, free_pages, n_free, ctx->d_ticket, ctx->d_status));
    cb_count_launch(1);
    return CB_OK;
}

extern "C" cb_status cb_slot_map(cb_ctx* ctx, const cb_slot_map_args* a, void* stream) {
    CB_CHECK_ARG(ctx && a);
    CB_CHECK_ARG(a->q_start && a->ctx_len && a->block_table && a->max_pages >= 1 && a->num_pages >= 1 && a->n_rows >= 0);
    if (a->n_rows == 0) return CB_OK;
    CB_CHECK_ARG(a->slots && a->positions && a->seqs);
    const cb_config& c = ctx->cfg;
    const unsigned blocks = (unsigned)(((long long)a->n_rows + kSlotThreads - 1) / kSlotThreads) + 1;
    CB_CUDA(cb_launch_pdl(cb_slot_map_kernel, dim3(blocks), dim3(kSlotThreads), 0, (cudaStream_t)stream, (int)c.batch, (int)c.page_size, (int)a->max_pages,
                          (int)a->num_pages, (int)a->n_rows, a->q_start, a->ctx_len, a->block_table, a->slots, a->positions, a->seqs, ctx->d_status));
    cb_count_launch(1);
    return CB_OK;
}
