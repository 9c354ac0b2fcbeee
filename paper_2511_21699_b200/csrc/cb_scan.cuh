// Sums over the sequences of a batch, by a block: where a flat list of what all of them need starts for each.
#pragma once
#include "cb_common.cuh"

#define CB_SUM_CAP (1u << 30)                                 // sums stop here: a cap only ever says "too much"
__device__ __forceinline__ uint32_t cb_add_capped(uint32_t a, uint32_t b) { return min(a + b, CB_SUM_CAP); }
__device__ __forceinline__ uint32_t cb_warp_sums(uint32_t x, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(CB_FULL, x, o); if (lane >= o) x = cb_add_capped(x, y); }
    return x;
}
// Inclusive sums of COUNTS counts over b < B in the block's shared memory: count(b, c) gives them (0 .. CB_SUM_CAP each), sums[k * B + b] holds what there is up to and
// with b.  NT threads, all of them; scratch: COUNTS * NT / 32 words.  Ends with a barrier.
template <int NT, int COUNTS, typename Count>
__device__ __forceinline__ void cb_block_sums(int B, uint32_t* sums, uint32_t* scratch, Count&& count) {
    constexpr int W = NT / 32;
    static_assert(W <= 32, "a warp sums the warps");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t base[COUNTS] = {};
    for (int b0 = 0; b0 < B; b0 += NT) {
        const int b = b0 + tid;
        uint32_t x[COUNTS] = {};
        if (b < B) count(b, x);
#pragma unroll
        for (int k = 0; k < COUNTS; ++k) {
            x[k] = cb_warp_sums(x[k], lane);
            if (lane == 31) scratch[k * W + warp] = x[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < COUNTS; ++k) {
            const uint32_t w = cb_warp_sums(lane < W ? scratch[k * W + lane] : 0u, lane);
            const uint32_t before = warp > 0 ? __shfl_sync(CB_FULL, w, warp - 1) : 0u;
            if (b < B) sums[k * B + b] = cb_add_capped(cb_add_capped(base[k], before), x[k]);
            base[k] = cb_add_capped(base[k], __shfl_sync(CB_FULL, w, W - 1));
        }
        __syncthreads();
    }
}
// The first b < B with sums[b] > x (B if there is none).
__device__ __forceinline__ int cb_upper(const uint32_t* sums, int B, uint32_t x) {
    int lo = 0, n = B;
    while (n > 0) {
        const int h = n >> 1;
        if (sums[lo + h] > x) n = h;
        else { lo += h + 1; n -= h + 1; }
    }
    return lo;
}
