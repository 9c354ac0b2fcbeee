// Log probabilities of given tokens, entropy and the best alternatives (cb_logprobs, cb_accept_logprobs).
//
// One pass over a row keeps, per thread, its running maximum m, s = sum e^d and t = sum e^d d with d = x - m; both sums are put on a new
// maximum when one comes.  The threads' (m, s, t) then go on the row's maximum M: log Z = M + log s, the token's log probability is
// (x - M) - log s, the entropy log s - t / s (two terms that are not negative, so nothing cancels).
//
// The alternatives need no second pass over the row.  Elements are ordered by value, equal ones by falling id (a 64-bit key).  Every
// thread knows its largest element; the K-th largest of these is a bound that at least K elements reach, and only the K threads above it
// can hold any that do.  So those K threads' elements, some 1/13 of a row for K = 20, are looked at once more (they are in L2), what reaches
// the bound is listed, usually little more than K elements, and the list is ranked by counting.
#include <math.h>

#include "cb_common.cuh"

namespace {

constexpr int kThreads = 256, kUnroll = 4, kWarps = kThreads / 32;
constexpr int kCand = 1024;                                   // elements listed; more than that are taken one after the other

struct LogprobParams {
    const void* logits;
    long long row_stride;
    const int32_t *rows, *tokens, *accept_nodes;
    float *logprobs, *entropy, *top_logprobs;
    int32_t* top_ids;
    int n_rows, n_out, V, K, T, Dmax;
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

template <bool BF16, bool TOP>
__global__ void __launch_bounds__(kThreads) cb_logprobs_kernel(const LogprobParams p) {
    CB_PDL_ENTRY();
    constexpr int E = Row<BF16>::E;
    __shared__ Stat s_stat[kWarps];
    __shared__ unsigned long long s_key[TOP ? kThreads : 1], s_cand[TOP ? kCand : 1], s_bound, s_best[kWarps];
    __shared__ int s_list[CB_MAX_TOP], s_lists, s_count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int i = blockIdx.x;
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
    if (pad || bad) {
        if (bad && !pad && tid == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_INVALID_ARG);
        if (tid == 0) {
            if (p.logprobs && p.tokens) p.logprobs[i] = 0.f;
            if (p.entropy) p.entropy[i] = 0.f;
        }
        if (TOP && tid < p.K) { p.top_ids[(size_t)i * p.K + tid] = -1; p.top_logprobs[(size_t)i * p.K + tid] = 0.f; }
        return;
    }
    const Row<BF16> r(p.logits, (long long)row * p.row_stride, p.V);
    const float x_tok = p.tokens && p.logprobs ? r.at(tok) : 0.f;

    Stat a = {-INFINITY, 0.f, 0.f};
    int best = 0;                                             // step at which the thread's largest element of a piece came
    for (int k0 = tid, step = 0; k0 < r.pieces; k0 += kThreads * kUnroll, ++step) {
        uint4 u[kUnroll];
        const uint32_t none = BF16 ? 0xFF80FF80u : 0xFF800000u;
#pragma unroll
        for (int q = 0; q < kUnroll; ++q) u[q] = k0 + q * kThreads < r.pieces ? r.piece(k0 + q * kThreads) : make_uint4(none, none, none, none);
        float m = -INFINITY;
#pragma unroll
        for (int q = 0; q < kUnroll; ++q) {
            float x[E];
            unpack<BF16>(u[q], x);
#pragma unroll
            for (int j = 0; j < E; ++j) m = fmaxf(m, x[j]);
        }
        if (m > a.m) {
            best = step;
            shift(a, m);
        }
        const float ref = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
        for (int q = 0; q < kUnroll; ++q) {
            float x[E];
            unpack<BF16>(u[q], x);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float d = max_keep_nan(x[j] - ref, -3e38f), e = ex2_approx(d * kLog2e);     // e = 0 times -inf would be NaN
                a.s += e;
                a.t = fmaf(e, d, a.t);
            }
        }
    }
    const float top_m = a.m;
    const int odds = r.head + r.tail;                         // at most 14 elements outside the pieces
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
    unsigned long long mine = 0;
    if constexpr (TOP) {
        // this thread's largest element, the lowest id among equal ones
        const int k0 = tid + best * kThreads * kUnroll;
        for (int q = 0; q < kUnroll && mine == 0; ++q) {
            const int k = k0 + q * kThreads;
            if (k >= r.pieces) break;
            float x[E];
            unpack<BF16>(r.piece(k), x);
#pragma unroll
            for (int j = E - 1; j >= 0; --j)
                if (x[j] == top_m) mine = key_of(x[j], r.id(k, j));
        }
        s_key[tid] = mine;
        if (tid == 0) { s_bound = 0; s_count = 0; s_lists = 0; }
    }
    __syncthreads();
    a = s_stat[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) a = join(a, s_stat[w]);
    const float log_s = a.m == -INFINITY ? NAN : logf(a.s);
    if (tid == 0) {
        if (p.tokens && p.logprobs) p.logprobs[i] = (x_tok - a.m) - log_s;
        if (p.entropy) p.entropy[i] = log_s - a.t / a.s;
    }
    if constexpr (TOP) {
        // the K threads with the largest elements, and the K-th of those
        int rank = 0;
        for (int k = 0; k < kThreads; ++k) rank += s_key[k] > mine;
        if (mine != 0 && rank < p.K) {
            s_list[rank] = tid;
            if (rank == p.K - 1) s_bound = mine;
            atomicAdd(&s_lists, 1);
        }
        __syncthreads();
        const unsigned long long bound = s_bound;
        const int lists = s_lists;
        auto list = [&](unsigned long long k) {
            if (k < bound) return;
            const int at = atomicAdd(&s_count, 1);
            if (at < kCand) s_cand[at] = k;
        };
        for (int l = warp; l < lists; l += kWarps)
            for (int k = s_list[l] + lane * kThreads; k < r.pieces; k += 32 * kThreads) {
                float x[E];
                unpack<BF16>(r.piece(k), x);
#pragma unroll
                for (int j = 0; j < E; ++j) list(key_of(x[j], r.id(k, j)));
            }
        const unsigned long long odd_key = my_odd >= 0 ? key_of(x_odd, my_odd) : 0;
        if (my_odd >= 0) list(odd_key);
        __syncthreads();
        const int count = s_count, found = min(count, p.K);
        int32_t* const ids = p.top_ids + (size_t)i * p.K;
        float* const lps = p.top_logprobs + (size_t)i * p.K;
        auto put = [&](int at, unsigned long long k) {
            ids[at] = id_of(k);
            lps[at] = (value_of(k) - a.m) - log_s;
        };
        if (count <= kCand) {
            for (int c = tid; c < count; c += kThreads) {
                const unsigned long long k = s_cand[c];
                int at = 0;
                for (int o = 0; o < count; ++o) at += s_cand[o] > k;
                if (at < p.K) put(at, k);
            }
        } else {
            // a few threads' elements make up much of what is large (a sorted row, say): one after the other
            unsigned long long last = ~0ull;
            for (int at = 0; at < found; ++at) {
                unsigned long long k1 = odd_key < last ? odd_key : 0;
                for (int l = warp; l < lists; l += kWarps)
                    for (int k = s_list[l] + lane * kThreads; k < r.pieces; k += 32 * kThreads) {
                        float x[E];
                        unpack<BF16>(r.piece(k), x);
#pragma unroll
                        for (int j = 0; j < E; ++j) {
                            const unsigned long long c = key_of(x[j], r.id(k, j));
                            if (c < last && c > k1) k1 = c;
                        }
                    }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) k1 = max(k1, __shfl_xor_sync(CB_FULL, k1, o));
                if (lane == 0) s_best[warp] = k1;
                __syncthreads();
                for (int w = 0; w < kWarps; ++w) k1 = max(k1, s_best[w]);
                last = k1;
                if (tid == 0) put(at, k1);
                __syncthreads();
            }
        }
        if (tid >= found && tid < p.K) { ids[tid] = -1; lps[tid] = -INFINITY; }
    }
}

cb_status launch_logprobs(const cb_logprobs_args& a, const LogprobParams& p, cudaStream_t st) {
    const bool f32 = a.logits_dtype == CB_DTYPE_F32;
    auto kernel = p.K ? (f32 ? cb_logprobs_kernel<false, true> : cb_logprobs_kernel<true, true>)
                      : (f32 ? cb_logprobs_kernel<false, false> : cb_logprobs_kernel<true, false>);
    CB_CUDA(cb_launch_pdl(kernel, dim3((unsigned)p.n_out), dim3(kThreads), 0, st, p));
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
    return launch_logprobs(*a, p, (cudaStream_t)stream);
}

extern "C" cb_status cb_accept_logprobs(cb_ctx* ctx, const int32_t* accept_nodes, const int32_t* out_tokens, const cb_logprobs_args* a, void* stream) {
    CB_CHECK_ARG(args_ok(ctx, a));
    CB_CHECK_ARG(accept_nodes && out_tokens);
    LogprobParams p = params_of(ctx, *a);
    p.accept_nodes = accept_nodes; p.tokens = out_tokens;
    p.n_out = ctx->cfg.batch * (ctx->cfg.max_depth + 1);
    return launch_logprobs(*a, p, (cudaStream_t)stream);
}
