// Log probabilities of given tokens, entropy and the best alternatives (cb_logprobs, cb_accept_logprobs).
//
// One pass over a row keeps, per thread, its running maximum m, s = sum e^d and t = sum e^d d with d = x - m; both sums are put on a new
// maximum when one comes.  The threads' (m, s, t) then go on the row's maximum M: log Z = M + log s, the token's log probability is
// (x - M) - log s, the entropy log s - t / s (two terms that are not negative, so nothing cancels).
//
// The alternatives need no second pass over the row.  Every thread notes the largest element of each of its steps, which it computes anyway.  At least K
// elements reach the K-th largest of 32 groups of threads' largest elements, and steps whose largest does are few (some 30 for K = 20); only
// those 64 bytes each are looked at once more, what reaches the bound is listed as a key (value, then falling id), little more than K elements as a rule,
// and the list is ranked by counting.  Where too many are as large as the bound (a constant row, or fewer than K tokens that are not forbidden), the list
// has those above it, and the lowest ids among the equal ones follow in order.  (Keys of all threads ranked, their elements all looked at again:
// 12 k cycles beside the 11 k of a row of 32 k bf16 logits.)
//
// A row is one CTA's, or, where that leaves SMs idle, a cluster's, whose CTAs take equal parts of it and hand their sums and their K best
// to the first one through distributed shared memory.
//
// 2,048 rows of 128 k bf16: 87 us, 6.0 TB/s of the 6.5 that a copy reaches (103 us in long runs at the clock that the power cap leaves: the
// exponential unit, an element each, is 72% busy); with 20 alternatives 111.  300 rows of 50 k fp32 with 20: 24 us (15 without).  Nine rows of 32 k bf16 with 5: 6.7.
#include <math.h>

#include "cb_common.cuh"

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;         // (512 threads a row: 5% faster for some shapes, 50% slower for others)
constexpr int kUnroll = 4;                                    // 16-byte pieces of a thread at a time
constexpr int kStep = kThreads * kUnroll;                     // and of the CTA
constexpr int kGroup = kThreads / 32;                         // threads of one of 32 groups
constexpr int kCand = 1024;                                   // elements listed at most
constexpr int kSlots = 32, kBlocks = 1024;                    // noted maxima of a thread; (thread, slot) blocks looked at again at most

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// The same place in another CTA of the cluster, and loads from there.
__device__ __forceinline__ uint32_t cluster_addr(uint32_t local, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
    return r;
}
__device__ __forceinline__ float ld_cluster_f(uint32_t a) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ unsigned long long ld_cluster_u64(uint32_t a) {
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}

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
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

struct LogprobParams {
    const void* logits;
    long long row_stride;
    const int32_t *rows, *tokens, *accept_nodes;
    float *logprobs, *entropy, *top_logprobs;
    int32_t* top_ids;
    int n_rows, n_out, V, K, T, Dmax;
    int cs;                                                   // CTAs per row
    uint32_t* status;
};

__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_keep_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
constexpr float kLog2e = 1.4426950408889634f;

// Running maximum and the sums relative to it.
struct Stat { float m, s, t; };
__device__ __forceinline__ void shift(Stat& a, float m) {     // onto a maximum that is no smaller
    if (a.m == -INFINITY) { a.m = m; return; }                // nothing yet (or NaN, which stays)
    const float d = a.m - m, w = ex2_approx(d * kLog2e);
    a.t = w > 0.f ? w * fmaf(a.s, d, a.t) : 0.f;              // (s d may be infinite where w is 0)
    a.s *= w;
    a.m = m;
}
__device__ __forceinline__ Stat join(Stat a, Stat b) {
    const float m = fmaxf(a.m, b.m);
    if (a.m < m) shift(a, m);
    if (b.m < m) shift(b, m);
    return {m, a.s + b.s, a.t + b.t};
}

// Order of the alternatives: the larger value first, equal ones by rising id.  0: no element.
__device__ __forceinline__ unsigned long long key_of(float x, uint32_t id) {
    const uint32_t u = __float_as_uint(x + 0.0f);             // -0 counts as 0
    return (unsigned long long)(u >> 31 ? ~u : u | 0x80000000u) << 32 | (0xFFFFFFFFu - id);
}
__device__ __forceinline__ float value_of(unsigned long long k) {
    const uint32_t u = (uint32_t)(k >> 32);
    return __uint_as_float(u >> 31 ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ int id_of(unsigned long long k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

template <bool BF16>
struct Row {
    static constexpr int E = BF16 ? 8 : 4;                    // elements of a 16-byte piece
    const char* base;
    int head, pieces, tail;                                   // elements before the first aligned piece, pieces, elements behind the last
    __device__ __forceinline__ Row(const void* logits, long long offset, int V) {
        base = (const char*)logits + offset * (BF16 ? 2 : 4);
        head = min((int)((16 - ((uintptr_t)base & 15)) & 15) / (BF16 ? 2 : 4), V);
        pieces = (V - head) / E;
        tail = V - head - pieces * E;
    }
    __device__ __forceinline__ float at(int i) const {
        if (BF16) return __uint_as_float((uint32_t)__ldg(reinterpret_cast<const unsigned short*>(base) + i) << 16);
        return __ldg(reinterpret_cast<const float*>(base) + i);
    }
    __device__ __forceinline__ uint4 piece(int k) const { return __ldg(reinterpret_cast<const uint4*>(base + head * (BF16 ? 2 : 4)) + k); }
    __device__ __forceinline__ int id(int k, int j) const { return head + k * E + j; }
    // the k-th of the elements that belong to no piece
    __device__ __forceinline__ int odd(int k) const { return k < head ? k : head + pieces * E + k - head; }
};
template <bool BF16>
__device__ __forceinline__ void unpack(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF16) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
        else x[i] = __uint_as_float(w[i]);
    }
}

template <bool BF16>
struct Block { uint4 u[kUnroll]; };                           // what a thread holds of a step
template <bool BF16>
__device__ __forceinline__ void load_block(Block<BF16>& b, const Row<BF16>& r, int k0, int end) {
    const uint32_t none = BF16 ? 0xFF80FF80u : 0xFF800000u;   // -inf
#pragma unroll
    for (int q = 0; q < kUnroll; ++q) b.u[q] = k0 + q * kThreads < end ? r.piece(k0 + q * kThreads) : make_uint4(none, none, none, none);
}
// Largest and smallest element; NaN is passed over.
template <bool BF16>
__device__ __forceinline__ void extremes(const Block<BF16>& b, float& hi, float& lo) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(b.u);
    if constexpr (BF16) {
        __nv_bfloat162 h = *reinterpret_cast<const __nv_bfloat162*>(w), l = h;
#pragma unroll
        for (int i = 1; i < 4 * kUnroll; ++i) {
            const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(w + i);
            h = __hmax2(h, x);
            l = __hmin2(l, x);
        }
        hi = fmaxf(__low2float(h), __high2float(h));
        lo = fminf(__low2float(l), __high2float(l));
    } else {
        hi = -INFINITY; lo = INFINITY;
#pragma unroll
        for (int i = 0; i < 4 * kUnroll; i += 2) {
            const float x = __uint_as_float(w[i]), y = __uint_as_float(w[i + 1]);
            asm("max.f32 %0, %0, %1, %2;" : "+f"(hi) : "f"(x), "f"(y));
            asm("min.f32 %0, %0, %1, %2;" : "+f"(lo) : "f"(x), "f"(y));
        }
    }
}
// Adds a block to s and t on reference ref.  CLAMP: some x - ref may be -inf (a forbidden token, or finite logits further apart than fp32 reaches, such as a
// mask of the type's lowest value beside a large one), whose e d = 0 * -inf must not be NaN.
template <bool BF16, bool CLAMP>
__device__ __forceinline__ void add_block(const Block<BF16>& b, float ref, uint64_t& s2, uint64_t& t2) {
    const uint64_t neg = f2_pack(-ref, -ref), l2e = f2_pack(kLog2e, kLog2e);
    const uint32_t* w = reinterpret_cast<const uint32_t*>(b.u);
#pragma unroll
    for (int i = 0; i < (BF16 ? 4 : 2) * kUnroll; ++i) {
        uint64_t d = BF16 ? f2_pack(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u))
                          : f2_pack(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        d = f2_add(d, neg);
        float a, c;
        if (CLAMP) {
            f2_unpack(d, a, c);
            d = f2_pack(max_keep_nan(a, -3e38f), max_keep_nan(c, -3e38f));
        }
        f2_unpack(f2_mul(d, l2e), a, c);
        const uint64_t e = f2_pack(ex2_approx(a), ex2_approx(c));
        s2 = f2_add(s2, e);
        t2 = f2_fma(e, d, t2);
    }
}

template <bool BF16, bool TOP>
__global__ void __launch_bounds__(kThreads, 4) cb_logprobs_kernel(const LogprobParams p) {
    CB_PDL_ENTRY();
    constexpr int E = Row<BF16>::E;
    __shared__ Stat s_stat[kWarps], s_all;
    __shared__ unsigned long long s_cand[TOP ? kCand : 1], s_best[kWarps], s_top[TOP ? CB_MAX_TOP : 1];
    __shared__ float s_hi[TOP ? kSlots : 1][TOP ? kThreads : 1], s_group[32];
    __shared__ unsigned short s_block[TOP ? kBlocks : 1];
    __shared__ int s_blocks, s_count, s_equal[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int i = blockIdx.x / p.cs, part = blockIdx.x - i * p.cs;          // the row's output, and which part of the row is this CTA's
    int row = i, tok = p.tokens ? p.tokens[i] : 0;
    bool pad = tok < 0, bad = tok >= p.V;
    if (p.accept_nodes) {
        const int b = i / (p.Dmax + 1), j = i - b * (p.Dmax + 1);
        const int node = j == 0 ? 0 : p.accept_nodes[(size_t)b * p.Dmax + j - 1];
        bad = bad || node < 0 || node >= p.T;
        row = b * p.T + node;
    } else {
        if (p.rows) row = p.rows[i];
        pad = pad || row < 0;
        bad = bad || row >= p.n_rows;
    }
    if (pad || bad) {                                         // the whole cluster
        if (part > 0) return;
        if (bad && !pad && tid == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
        if (tid == 0) {
            if (p.logprobs && p.tokens) p.logprobs[i] = 0.f;
            if (p.entropy) p.entropy[i] = 0.f;
        }
        if (TOP && tid < p.K) { p.top_ids[(size_t)i * p.K + tid] = -1; p.top_logprobs[(size_t)i * p.K + tid] = 0.f; }
        return;
    }
    const Row<BF16> r(p.logits, (long long)row * p.row_stride, p.V);
    const float x_tok = part == 0 && p.tokens && p.logprobs ? r.at(tok) : 0.f;
    const int per = (r.pieces + p.cs - 1) / p.cs, begin = min(part * per, r.pieces), end = min(begin + per, r.pieces);

    float ref = -INFINITY;                                    // the thread's running maximum
    uint64_t s2 = 0, t2 = 0;                                  // two sums each
    // alternatives: the largest element of every so many steps
    const int steps = (end - begin + kStep - 1) / kStep, per_slot = (steps + kSlots - 1) / kSlots;
    int slots = 0, in_slot = 0;
    float slot_hi = -INFINITY;
    Block<BF16> cur, next;                                    // (three steps in shared memory, by bulk copies, were no faster than one ahead in registers)
    load_block(cur, r, begin + tid, end);
    for (int k0 = begin + tid; k0 < end; k0 += kStep) {
        load_block(next, r, k0 + kStep, end);
        float hi, lo;
        extremes(cur, hi, lo);
        if (hi > ref) {                                       // -inf: nothing yet (or NaN, which stays)
            if (ref > -INFINITY) {
                const float d = ref - hi, w = ex2_approx(d * kLog2e);
                float s0, s1, t0, t1;
                f2_unpack(s2, s0, s1);
                f2_unpack(t2, t0, t1);
                t2 = w > 0.f ? f2_pack(w * fmaf(s0, d, t0), w * fmaf(s1, d, t1)) : 0;      // (s d may be infinite where w is 0)
                s2 = f2_pack(s0 * w, s1 * w);
            }
            ref = hi;
        }
        if constexpr (TOP) {
            slot_hi = fmaxf(slot_hi, hi);
            if (++in_slot == per_slot) { s_hi[slots++][tid] = slot_hi; slot_hi = -INFINITY; in_slot = 0; }
        }
        const float base = ref == -INFINITY ? 0.f : ref;
        if (lo - base == -INFINITY) add_block<BF16, true>(cur, base, s2, t2);
        else add_block<BF16, false>(cur, base, s2, t2);
        cur = next;
    }
    Stat a;
    {
        float s0, s1, t0, t1;
        f2_unpack(s2, s0, s1);
        f2_unpack(t2, t0, t1);
        a = {ref, s0 + s1, t0 + t1};
    }
    const int odds = part == 0 ? r.head + r.tail : 0;         // at most 14 elements outside the pieces: the first CTA's
    const int my_odd = tid < odds ? r.odd(tid) : -1;
    const float x_odd = my_odd >= 0 ? r.at(my_odd) : -INFINITY;
    if (my_odd >= 0) {
        const Stat o = x_odd == -INFINITY ? Stat{-INFINITY, 0.f, 0.f} : Stat{x_odd, x_odd < INFINITY ? 1.f : NAN, 0.f};
        a = join(a, o);
        if (x_odd != x_odd) a.s = NAN;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a = join(a, {__shfl_xor_sync(CB_FULL, a.m, o), __shfl_xor_sync(CB_FULL, a.s, o), __shfl_xor_sync(CB_FULL, a.t, o)});
    if (lane == 0) s_stat[warp] = a;
    if constexpr (TOP) {
        if (in_slot) s_hi[slots++][tid] = slot_hi;
        float group = ref;
#pragma unroll
        for (int o = 1; o < kGroup; o <<= 1) group = fmaxf(group, __shfl_xor_sync(CB_FULL, group, o));
        if (lane % kGroup == 0) s_group[tid / kGroup] = group;
        if (tid == 0) s_blocks = s_count = 0;
    }
    __syncthreads();
    if (warp == 0) {                                          // the CTA's sums; only this warp writes any result
        a = s_stat[lane % kWarps];
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1) a = join(a, {__shfl_xor_sync(CB_FULL, a.m, o), __shfl_xor_sync(CB_FULL, a.s, o), __shfl_xor_sync(CB_FULL, a.t, o)});
        if (lane == 0) s_all = a;
    }
    if constexpr (TOP) {
        // the bound, in every warp: the K-th largest of the groups' (equal ones by number)
        const float mine = s_group[lane];
        int rank = 0;
#pragma unroll
        for (int o = 0; o < 32; ++o) rank += s_group[o] > mine || (s_group[o] == mine && o < lane);
        const float bound = __shfl_sync(CB_FULL, mine, __ffs(__ballot_sync(CB_FULL, rank == p.K - 1)) - 1);
        // Lists the elements that reach the bound, or lie above it, as keys; false: there are too many.
        auto collect = [&](bool above) {
            auto in = [&](float x) { return above ? x > bound : x >= bound; };
            auto list = [&](unsigned long long k) {
                const int at = atomicAdd(&s_count, 1);
                if (at < kCand) s_cand[at] = k;
            };
            for (int k = 0; k < slots; ++k)
                if (in(s_hi[k][tid])) {
                    const int at = atomicAdd(&s_blocks, 1);
                    if (at < kBlocks) s_block[at] = (unsigned short)(k * kThreads + tid);
                }
            __syncthreads();
            const int blocks = s_blocks;
            if (blocks > kBlocks) return false;
            // all their pieces dealt to the threads, four loads at a time
            const int pieces = per_slot * kUnroll, all = blocks * pieces;
            for (int w0 = tid; w0 < all; w0 += 4 * kThreads) {
                int at[4];
                uint4 u[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int w = w0 + q * kThreads, b = per_slot == 1 ? w / kUnroll : w / pieces, r4 = w - b * pieces;
                    at[q] = end;
                    if (w < all) {
                        const int block = s_block[b];
                        at[q] = begin + (block / kThreads * per_slot + r4 / kUnroll) * kStep + r4 % kUnroll * kThreads + block % kThreads;
                    }
                    if (at[q] < end) u[q] = r.piece(at[q]);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (at[q] >= end) continue;
                    float x[E], hi = -INFINITY;
                    unpack<BF16>(u[q], x);
#pragma unroll
                    for (int j = 0; j < E; ++j) hi = fmaxf(hi, x[j]);
                    if (!in(hi)) continue;                    // most pieces
#pragma unroll
                    for (int j = 0; j < E; ++j)
                        if (in(x[j])) list(key_of(x[j], r.id(at[q], j)));
                }
            }
            if (my_odd >= 0 && in(x_odd)) list(key_of(x_odd, my_odd));
            __syncthreads();
            return s_count <= kCand;
        };
        bool listed = collect(false), equals = false;
        if (!listed) {
            __syncthreads();
            if (tid == 0) s_blocks = s_count = 0;
            __syncthreads();
            listed = collect(true);
            equals = true;
        }
        int found = 0;
        if (listed) {
            const int count = s_count;
            found = min(count, p.K);
            for (int c = tid; c < count; c += kThreads) {
                const unsigned long long k = s_cand[c];
                int at = 0;
                for (int o = 0; o < count; ++o) at += s_cand[o] > k;
                if (at < p.K) s_top[at] = k;
            }
            // the bound's equals in the order of their ids: what lies before the pieces, the pieces, 256 at a time, what lies behind them
            for (int k0 = begin - kThreads; equals && found < p.K && k0 < end + kThreads; k0 += kThreads) {
                const bool head = k0 < begin, tail = k0 >= end;
                const int k = k0 + tid;
                uint32_t equal = 0;                           // which of this thread's elements
                if (head || tail) {
                    const int o = head ? tid : r.head + tid;
                    if (part == 0 && o < (head ? r.head : r.head + r.tail)) equal = r.at(r.odd(o)) == bound;
                } else if (k < end) {
                    float x[E];
                    unpack<BF16>(r.piece(k), x);
#pragma unroll
                    for (int j = 0; j < E; ++j) equal |= (uint32_t)(x[j] == bound) << j;
                }
                int before = __popc(equal);
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int t = __shfl_up_sync(CB_FULL, before, o);
                    if (lane >= o) before += t;
                }
                if (lane == 31) s_equal[warp] = before;
                before -= __popc(equal);
                __syncthreads();
                int total = 0;
                for (int w = 0; w < kWarps; ++w) {
                    if (w < warp) before += s_equal[w];
                    total += s_equal[w];
                }
                for (int at = found + before; equal != 0 && at < p.K; ++at) {
                    const int j = __ffs(equal) - 1;
                    equal &= equal - 1;
                    s_top[at] = key_of(bound, head ? r.odd(tid) : (tail ? r.odd(r.head + tid) : r.id(k, j)));
                }
                found = min(found + total, p.K);
                __syncthreads();
            }
        } else {
            // thousands above the bound too (a few threads' elements make up what is large, as in a sorted row): one after the other
            unsigned long long last = ~0ull;
            while (found < p.K) {
                unsigned long long k1 = 0;
                if (my_odd >= 0 && x_odd == x_odd && key_of(x_odd, my_odd) < last) k1 = key_of(x_odd, my_odd);
                for (int k = begin + tid; k < end; k += kThreads) {
                    float x[E];
                    unpack<BF16>(r.piece(k), x);
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const unsigned long long c = x[j] == x[j] ? key_of(x[j], r.id(k, j)) : 0;
                        if (c < last && c > k1) k1 = c;
                    }
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) k1 = max(k1, __shfl_xor_sync(CB_FULL, k1, o));
                if (lane == 0) s_best[warp] = k1;
                __syncthreads();
                for (int w = 0; w < kWarps; ++w) k1 = max(k1, s_best[w]);
                if (tid == 0) s_top[found] = k1;
                __syncthreads();
                if (k1 == 0) break;
                last = k1;
                ++found;
            }
        }
        if (tid >= found && tid < p.K) s_top[tid] = 0;        // (places that nobody has written)
    }
    if (p.cs > 1) {
        // The first CTA reads what the others have; they stay until it has.
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (part == 0) {
            if (warp == 0) {
                const uint32_t o = cluster_addr(smem_u32(&s_all), (uint32_t)(lane % p.cs));      // a power of two
                a = {ld_cluster_f(o), ld_cluster_f(o + 4), ld_cluster_f(o + 8)};
                for (int d = p.cs / 2; d > 0; d >>= 1) a = join(a, {__shfl_xor_sync(CB_FULL, a.m, d), __shfl_xor_sync(CB_FULL, a.s, d), __shfl_xor_sync(CB_FULL, a.t, d)});
            }
            if constexpr (TOP) {
                const int n = p.cs * p.K;                     // at most 8 lists of 32
                for (int k = tid; k < n; k += kThreads) s_cand[k] = ld_cluster_u64(cluster_addr(smem_u32(&s_top[k % p.K]), (uint32_t)(k / p.K)));
                __syncthreads();
                unsigned long long k = 0;
                int rank = 0;
                if (tid < n) {
                    k = s_cand[tid];
                    for (int o = 0; o < n; ++o) rank += s_cand[o] > k;
                }
                __syncthreads();
                if (tid < p.K) s_top[tid] = 0;
                __syncthreads();
                if (k != 0 && rank < p.K) s_top[rank] = k;
            }
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        if (part > 0) {
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            return;
        }
    }
    const float log_s = a.m == -INFINITY ? NAN : logf(a.s);
    if (tid == 0) {
        if (p.tokens && p.logprobs) p.logprobs[i] = (x_tok - a.m) - log_s;
        if (p.entropy) p.entropy[i] = log_s - a.t / a.s;
    }
    if constexpr (TOP) {
        __syncthreads();
        if (tid < p.K) {
            const unsigned long long k = s_top[tid];
            p.top_ids[(size_t)i * p.K + tid] = k == 0 ? -1 : id_of(k);
            // no element for this place: the vocabulary is shorter, or what is left are NaNs
            p.top_logprobs[(size_t)i * p.K + tid] = k == 0 ? (tid < p.V ? NAN : -INFINITY) : (value_of(k) - a.m) - log_s;
        }
    }
    __syncwarp();
    if (p.cs > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// CTAs per row.  A cluster costs a launch some 0.3 us and every row the hand-over; it pays where rows alone leave SMs without work, and, with
// up to four CTAs an SM, where a row is so long that its CTA ends well after the rest.  Measured, us with 1, 2, 4, 8 CTAs a row:
//   9 rows of 128 k fp32 10.5, 7.5, 5.5, 4.4;  40 of 128 k bf16 12.7, 9.0, 7.0, 7.8;  75 of 50 k fp32 10.7, 8.3, 7.7, 9.8
//   150 of 128 k bf16 15.0, 16.5, 14.7, 16.8;  300 of 128 k bf16 27.5, 21.8, 23.2, 28.4;  300 of 50 k fp32 14.7, 18.5, 20.0, 24.6;  600 of 128 k 34.6, 35.0, 39.9, 52.7
//   with 20 alternatives 9 of 128 k bf16 14.4, 11.1, 8.8, 8.4;  40 16.1, 12.4, 11.5, 14.0;  150 of fp32 27.9, 24.8, 29.8, 37.0;  with five 9 of 32 k 6.6, 7.1, 6.5, 6.4
// Few rows around the shortest that are shared (none and 20 alternatives):
//   9 of 16 k fp32 3.3, 3.2, 2.8, 3.0 and 6.0, 6.3, 5.9, 6.7;  of 24 k 4.1, 3.8, 3.4, 3.2 and 7.0, 6.7, 6.6, 6.7;  of 32 k 4.7, 4.1, 3.4, 3.2 and 7.8, 7.2, 6.7, 6.8
//   of 48 k fp32 6.2, 4.8, 3.8, 3.5 and 9.5, 8.2, 7.0, 7.5;  of 64 k 7.5, 5.5, 4.1, 3.5 and 11.0, 9.1, 7.5, 7.4;  74 of 32 k fp32 7.5, 5.8, 6.0, 7.3 and 10.2, 8.9, 11.0, 16.7
//   9 of 24 k bf16 3.4, 3.7, 3.1, 3.3 and 6.5, 6.8, 6.5, 7.3;  of 32 k 3.8, 3.8, 3.3, 3.3 and 6.8, 7.0, 6.7, 7.3;  of 48 k 4.9, 4.2, 3.7, 3.2 and 8.3, 7.8, 7.2, 7.3
//   74 of 32 k bf16 3.9, 4.0, 5.5, 7.3 and 6.9, 7.3, 10.1, 17.2;  of 48 k 6.1, 5.0, 6.9, 7.5 and 9.1, 8.2, 12.1, 17.2
int pick_cluster(long long rows, int V, int K, int num_sms, bool f32) {
    int cs = 1;
    if (V < (f32 ? 24000 : 48000)) return cs;
    while (cs < 8) {
        const long long ctas = rows * cs * 2, each = V / (cs * 2);
        const bool idle = ctas * 10 <= 11ll * num_sms, room = ctas * 10 <= 42ll * num_sms;
        if (!(idle ? each >= (f32 ? 8000 : 12000) : room && each >= (K ? 64000 : 32000))) break;
        cs *= 2;
    }
    return cs;
}

cb_status launch_logprobs(const cb_logprobs_args& a, LogprobParams p, int num_sms, cudaStream_t st) {
    const bool f32 = a.logits_dtype == CB_DTYPE_F32;
    p.cs = pick_cluster(p.n_out, p.V, p.K, num_sms, f32);
    if ((long long)p.n_out * p.cs > 0x7FFFFFFFll) return CB_ERR_UNSUPPORTED;
    auto kernel = p.K ? (f32 ? cb_logprobs_kernel<false, true> : cb_logprobs_kernel<true, true>)
                      : (f32 ? cb_logprobs_kernel<false, false> : cb_logprobs_kernel<true, false>);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.n_out * p.cs)); cfg.blockDim = dim3(kThreads); cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)p.cs; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = p.cs > 1 ? 2 : 1;
    CB_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
    cb_count_launch(1);
    return CB_OK;
}

bool args_ok(const cb_ctx* ctx, const cb_logprobs_args* a) {
    if (!ctx || !a || !a->logits) return false;
    if (a->logits_dtype != CB_DTYPE_F32 && a->logits_dtype != CB_DTYPE_BF16) return false;
    if (a->logits_row_stride < ctx->cfg.vocab) return false;
    if ((uintptr_t)a->logits & (a->logits_dtype == CB_DTYPE_F32 ? 3 : 1)) return false;
    if (a->top_k < 0 || a->top_k > CB_MAX_TOP) return false;
    return a->top_k == 0 || (a->top_ids && a->top_logprobs);
}
LogprobParams params_of(cb_ctx* ctx, const cb_logprobs_args& a) {
    LogprobParams p = {};
    p.logits = a.logits; p.row_stride = a.logits_row_stride;
    p.logprobs = a.logprobs; p.entropy = a.entropy; p.top_ids = a.top_ids; p.top_logprobs = a.top_logprobs;
    p.V = ctx->cfg.vocab; p.K = a.top_k; p.T = ctx->cfg.max_nodes; p.Dmax = ctx->cfg.max_depth;
    p.status = ctx->d_status;
    return p;
}

}  // namespace

extern "C" cb_status cb_logprobs(cb_ctx* ctx, const cb_logprobs_args* a, void* stream) {
    CB_CHECK_ARG(args_ok(ctx, a));
    CB_CHECK_ARG(a->n_out >= 0 && a->n_rows >= 0 && (a->rows || a->n_out <= a->n_rows));
    if (a->n_out == 0) return CB_OK;
    LogprobParams p = params_of(ctx, *a);
    p.rows = a->rows; p.tokens = a->tokens; p.n_rows = a->n_rows; p.n_out = a->n_out;
    return launch_logprobs(*a, p, ctx->num_sms, (cudaStream_t)stream);
}

extern "C" cb_status cb_accept_logprobs(cb_ctx* ctx, const int32_t* accept_nodes, const int32_t* out_tokens, const cb_logprobs_args* a, void* stream) {
    CB_CHECK_ARG(args_ok(ctx, a));
    CB_CHECK_ARG(accept_nodes && out_tokens);
    LogprobParams p = params_of(ctx, *a);
    p.accept_nodes = accept_nodes; p.tokens = out_tokens;
    p.n_out = ctx->cfg.batch * (ctx->cfg.max_depth + 1);
    return launch_logprobs(*a, p, ctx->num_sms, (cudaStream_t)stream);
}
