// Launcher of chunk attention over all of the context (the kernel is in cb_chunk_tc.cuh).
#include "cb_chunk_tc.cuh"

cb_status cb_chunk_launch_tensor(cb_ctx* ctx, const CbChunkParams& given, cudaStream_t st) {
    CbChunkParams p = given;
    if (p.num_pages >= 1 << 29) return CB_ERR_UNSUPPORTED;   // (a page's coordinate is twice its number)
    chunk_split(ctx, p, p.max_keys);
    ChunkMaps maps;
    if (!encode_pool(&maps.k, p.k_pool, p) || !encode_pool(&maps.v, p.v_pool, p) || !encode_queries(&maps.q, p)) return CB_ERR_CUDA;
    return p.D == 128 ? launch_chunk<128>(p, maps, st, ctx->device) : launch_chunk<64>(p, maps, st, ctx->device);
}
