// Sums over the sequences of a batch, by a block: where a flat list of what all of them need starts for each.
#pragma once
#include "cb_common.cuh"

// Inclusive sums of two counts over b < B in the block's shared memory: count(b) gives both, and sum0[b], sum1[b] hold what there is up to and
// with b, capped at 2^31 - 1 (a cap only ever says "too much").  NT threads, all of them; scratch: 2 x 33 words.  Ends with a barrier.
template <int NT, typename Count>
__device__ __forceinline__ void cb_block_sums(int B, int32_t* sum0, int32_t* sum1, long long* scratch, Count&& count) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long base0 = 0, base1 = 0;
    for (int b0 = 0; b0 < B; b0 += NT) {
        const int b = b0 + tid;
        int c0 = 0, c1 = 0;
        if (b < B) count(b, &c0, &c1);
        long long x0 = c0, x1 = c1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y0 = __shfl_up_sync(CB_FULL, x0, o), y1 = __shfl_up_sync(CB_FULL, x1, o);
            if (lane >= o) { x0 += y0; x1 += y1; }
        }
        if (lane == 31) { scratch[warp] = x0; scratch[33 + warp] = x1; }
        __syncthreads();
        long long before0 = base0, before1 = base1;
        for (int w = 0; w < NT / 32; ++w) {
            const long long t0 = scratch[w], t1 = scratch[33 + w];
            if (w < warp) { before0 += t0; before1 += t1; }
            base0 += t0; base1 += t1;
        }
        if (b < B) {
            sum0[b] = (int32_t)min(before0 + x0, 0x7FFFFFFFll);
            sum1[b] = (int32_t)min(before1 + x1, 0x7FFFFFFFll);
        }
        __syncthreads();
    }
}
// The first b < B with sums[b] > x (B if there is none).
__device__ __forceinline__ int cb_upper(const int32_t* sums, int B, int x) {
    int lo = 0, n = B;
    while (n > 0) {
        const int h = n >> 1;
        if (sums[lo + h] > x) n = h;
        else { lo += h + 1; n -= h + 1; }
    }
    return lo;
}
