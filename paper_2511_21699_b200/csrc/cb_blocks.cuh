// Attention over selected blocks: what its kernels share.
#pragma once
#include "cb_chunk.cuh"

// The lists that attention over selected blocks reads: per sequence and kv head n_select numbers of blocks of 1 << shift tokens.
struct CbBlockLists {
    const int32_t* blocks;    // [batch, Hkv, n_select]; null: all of the context, no lists
    int n_select, shift;
};
// A sequence of ctx cached tokens as its rows see it: the selected blocks one behind the other, and what follows the context behind them.  All blocks but
// the newest, which is the last one of every list, are full, so that the number of visible tokens is the same for all heads.
__host__ __device__ __forceinline__ int cb_blocks_of(int ctx, int shift) { return (int)(((long long)ctx + (1ll << shift) - 1) >> shift); }
__host__ __device__ __forceinline__ int cb_seen(const CbBlockLists& l, int ctx) {
    const int nb = cb_blocks_of(ctx, l.shift);
    return nb > l.n_select ? ctx - ((nb - l.n_select) << l.shift) : ctx;
}
// Column of the block table for the i-th page that (b, kv head) sees, nb the blocks of the context; -1: none.
__device__ __forceinline__ int cb_page_column(const CbBlockLists& l, int b, int Hkv, int kh, int nb, int i) {
    const int per = l.shift - 4, at = i >> per, ns = min(nb, l.n_select);
    if (at >= ns) return (nb << per) + i - (ns << per);       // behind the context: the chunk's own tokens
    const int block = l.blocks[((size_t)b * Hkv + kh) * l.n_select + at];
    return block >= 0 && block < nb ? (block << per) + (i & ((1 << per) - 1)) : -1;
}

// What attention over selected blocks is given: of chunks, and of draft trees (rows b * T + node, max_chunk = T).
struct CbListParams : CbChunkParams {
    static constexpr int kMode = 1;
    CbBlockLists l;
};
struct CbListTreeParams : CbListParams {
    static constexpr int kMode = 2;
    const __nv_bfloat16 *k_tree, *v_tree;
    const uint32_t* mask;
    const int32_t* n_nodes;
    int T, W;
};
// Their sequences, the context as the rows see it.
__device__ __forceinline__ CbChunkSeq cb_chunk_seq(const CbListParams& p, int b) {
    CbChunkSeq s = cb_chunk_seq(static_cast<const CbChunkParams&>(p), b);
    if (s.n > 0) s.ctx = cb_seen(p.l, s.ctx);
    return s;
}
// Nodes of a tree, 0 where its lengths are out of their bounds, and what is wrong with them then (0: there are none).
__device__ __forceinline__ int cb_tree_nodes(const CbListTreeParams& p, int b) {
    const int n = p.n_nodes[b];
    return (uint32_t)n <= (uint32_t)p.T && (uint32_t)p.ctx_len[b] <= (uint32_t)p.max_keys ? n : 0;
}
__device__ __forceinline__ int cb_tree_error(const CbListTreeParams& p, int b) {
    const int n = p.n_nodes[b];
    if (n == 0 || cb_tree_nodes(p, b) > 0) return 0;
    return n > 0 && n <= p.T && p.ctx_len[b] > p.max_keys ? CB_ERR_KV_FULL : CB_ERR_INVALID_ARG;
}
// (Errors are looked for where rows of zeros are written: held through the walk over the units they cost 24 bytes of spills a thread, and 0.5 to 1% of the time.)
__device__ __forceinline__ CbChunkSeq cb_chunk_seq(const CbListTreeParams& p, int b) {
    return {b * p.T, cb_tree_nodes(p, b), cb_seen(p.l, p.ctx_len[b]), 0};
}

cb_status cb_block_launch_tensor(cb_ctx* ctx, const CbListParams& p, cudaStream_t st);
cb_status cb_block_launch_tensor(cb_ctx* ctx, const CbListTreeParams& p, cudaStream_t st);
// For units of up to 16 rows x heads: max_chunk * G <= 16.
cb_status cb_block_launch_token(cb_ctx* ctx, const CbListParams& p, cudaStream_t st);
