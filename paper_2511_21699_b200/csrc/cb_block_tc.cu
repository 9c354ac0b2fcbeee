// Launchers of attention over selected blocks on the tensor cores: chunk attention's kernel (cb_chunk_tc.cuh), whose copies find their pages through the
// lists, and whose rows may be a tree's nodes.  Measured with lists of 2,048 tokens, 64 query heads over 8 of 128: 8 chunks of 129 to 256 tokens 120 us in short runs, 142 in long
// ones (the dense call over as many keys takes the same); 16 trees of 64 nodes 84 and 99 (the dense tree call 75 in short runs; 94 and 112 bytes of spills a thread here, 132 and 148 there).
#include <algorithm>

#include "cb_chunk_tc.cuh"

namespace {

template <typename P, typename Encode>
cb_status launch(cb_ctx* ctx, const P& given, cudaStream_t st, long long own, Encode&& more) {
    P p = given;
    if (p.num_pages >= 1 << 29) return CB_ERR_UNSUPPORTED;   // (a page's coordinate is twice its number)
    chunk_split(ctx, p, std::min<long long>(p.max_keys, (long long)p.l.n_select << p.l.shift) + own);
    MapsOf<P> maps;
    if (!encode_pool(&maps.k, p.k_pool, p) || !encode_pool(&maps.v, p.v_pool, p) || !encode_queries(&maps.q, p) || !more(&maps)) return CB_ERR_CUDA;
    return p.D == 128 ? launch_chunk<128>(p, maps, st, ctx->device) : launch_chunk<64>(p, maps, st, ctx->device);
}

}  // namespace

cb_status cb_block_launch_tensor(cb_ctx* ctx, const CbListParams& p, cudaStream_t st) {
    return launch(ctx, p, st, p.max_chunk, [](ChunkMaps*) { return true; });
}
cb_status cb_block_launch_tensor(cb_ctx* ctx, const CbListTreeParams& p, cudaStream_t st) {
    return launch(ctx, p, st, CB_KT, [&](ChunkTreeMaps* m) { return encode_tree(&m->kt, p.k_tree, p) && encode_tree(&m->vt, p.v_tree, p); });
}
