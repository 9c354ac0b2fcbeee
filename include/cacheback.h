/*
 * cacheback.h — C ABI of the Cacheback draft-and-verify step on one NVIDIA B200 (sm_100a).
 *
 * One decoding step of Cacheback speculative decoding (paper Section 3) is, per sequence of a batch:
 *   cb_update      slide a window over the newly accepted tokens and insert every leader->follower pair
 *                  into the sequence's LRU cache table                       (Section 3.1; 3.2 last par.)
 *   cb_draft_tree  grow a draft token tree by recursive table queries, breadth first, and emit parent
 *                  indices, depths and the ancestor ("tree attention") mask  (Section 3.2)
 *   cb_tree_attn   let every tree token attend to the sequence's paged KV cache plus its tree ancestors
 *                  (the attention of the single verification forward pass)    (Section 3.2)
 *   cb_accept      take the target's greedy choice after every node and keep the longest verified
 *                  branch plus one more token                                 (Section 3.2)
 * Beside it: cb_chunk_append and cb_chunk_attn bring prompts and single tokens into the paged cache and attend over it, cb_tree_rope
 * makes the rotated queries and keys of a tree, cb_logprobs says how likely tokens were; cb_pages_assign and cb_slot_map keep the cache's block
 * tables on the GPU, cb_block_summary, cb_block_select, cb_block_attn and cb_block_tree_attn attend to the parts of a long context that matter.
 *
 * Conventions
 *   - Every tensor pointer is a DEVICE pointer owned by the caller unless a parameter says "host".
 *     The library never allocates or frees device memory: all of its state and scratch lives in the
 *     workspace handed to cb_create.
 *   - `stream` is a cudaStream_t passed as void*. The calls of a step, the ones beside it and cb_reset only enqueue work
 *     on it; they never synchronise.  Calls on one context must be ordered (same stream, or events).
 *   - Host-detectable argument errors are returned at once and nothing is enqueued.  Conditions only
 *     the device can see (a probe limit, a bounded wait that ran out) are recorded in a device status
 *     word; the kernel finishes cleanly and cb_poll_status reports the first such code.
 *   - Token ids are int32 >= 0; -1 is "no token".  Rows of per-node outputs beyond a sequence's node
 *     count are padded: tokens / parents / depths / accepted nodes / emitted tokens with -1, mask and
 *     attention rows with 0.
 *   - bf16 tensors are passed as void* (16-bit brain floats, row-major, last index fastest).
 */
#ifndef CACHEBACK_H_
#define CACHEBACK_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cb_ctx cb_ctx; /* opaque */

typedef enum {
    CB_OK = 0,
    CB_ERR_INVALID_ARG = 1,
    CB_ERR_WORKSPACE_TOO_SMALL = 2,
    CB_ERR_CUDA = 3,
    CB_ERR_PROBE_LIMIT = 4, /* device: a hash probe visited every bucket without finding a free slot  */
    CB_ERR_TIMEOUT = 5,     /* device: a bounded wait (mbarrier / flag) ran out                        */
    CB_ERR_UNSUPPORTED = 6,
    CB_ERR_STATIC_LIMIT = 7, /* cb_accept_static: the problem does not fit the built-in scratch array       */
    CB_ERR_KV_FULL = 8,      /* device: a sequence whose pages cannot hold its new tokens (cb_kv_commit, the calls beside the step) */
    CB_ERR_CANARY = 9        /* checking build only: a guard word beside a workspace region was overwritten    */
} cb_status;

enum { CB_DTYPE_F32 = 0, CB_DTYPE_BF16 = 1 };

/* cb_config.flags */
enum {
    CB_FLAG_NO_FOLLOWER_REFRESH = 1u, /* re-inserting a stored follower leaves its recency unchanged     */
    CB_FLAG_ATTN_CUDA_CORES = 2u,     /* run tree and chunk attention on plain CUDA-core kernels (debug aid) */
    CB_FLAG_ATTN_CTA_PAIRS = 4u       /* tree attention of multi-row-tile launches (head_dim 128) as pairs of
                                         CTAs issuing 2-CTA tensor-core products; measured slower than the
                                         default on the configurations benchmarked, kept as an alternative */
};

/*
 * Shape of one context. Table parameters follow Section 3.1 / 3.2:
 *   LL, FL  leader / follower length in tokens          (1..4, 1..8)
 *   LC, FC  leader capacity per sequence, follower capacity per leader   (1..2^20, 1..128)
 *   max_nodes  tree-size cap, root included: the paper's total draft length (TDL)   (1..128)
 *   crt        nodes reserved for query levels >= 2: level 1 fills at most max(1, max_nodes - crt)
 *   max_depth  deepest node depth allowed (root = 0)
 * Attention shape: n_q_heads % n_kv_heads == 0, head_dim in {64, 128}, page_size == 16.
 * vocab is the logits row length for cb_accept.
 */
typedef struct {
    int32_t batch;
    int32_t LL, FL, LC, FC;
    int32_t max_nodes, crt, max_depth;
    int32_t vocab;
    int32_t n_q_heads, n_kv_heads, head_dim, page_size;
    uint32_t flags;
} cb_config;

/* Bytes of device workspace cb_create needs for this shape (tables + scratch). Host call. */
cb_status cb_workspace_bytes(const cb_config* cfg, size_t* bytes);

/*
 * Creates a context over caller-owned device memory `dev_workspace` (256-byte aligned, `bytes` long,
 * on the current device) and empties every table.  Synchronises the device once.  *out is a small
 * host object; the workspace must outlive it and belongs to the library until cb_destroy.
 */
cb_status cb_create(const cb_config* cfg, void* dev_workspace, size_t bytes, cb_ctx** out);

/* Frees the host object only; never touches caller memory. NULL is allowed. */
void cb_destroy(cb_ctx* ctx);

/*
 * Empties the tables of the sequences whose entry in dev_seq_mask ([batch] int32, non-zero = reset) is
 * set, or of all sequences when dev_seq_mask is NULL (the per-task state reset of Section 4).
 */
cb_status cb_reset(cb_ctx* ctx, const int32_t* dev_seq_mask, void* stream);

/*
 * Table update (Section 3.1 insertion rules; Section 3.2, last paragraph: every leader-follower window that the newly
 * accepted tokens complete is inserted; Section 3.3 prompt initialisation = the same call with n_old = 0).
 *   tokens   int32 [batch, row_stride]  token history of every sequence
 *   n_old    int32 [batch]  tokens already ingested by earlier calls
 *   n_new    int32 [batch]  tokens valid now (n_new >= n_old; n_new <= row_stride)
 * For sequence b every complete window i (leader = tokens[i .. i+LL), follower = tokens[i+LL ..
 * i+LL+FL)) whose last token is new (i+LL+FL-1 in [n_old, n_new)) is inserted in increasing i:
 * the leader is created (evicting the least recently used leader with its followers when LC are
 * stored) or refreshed; the follower is appended (evicting the leader's least recently inserted
 * follower when FC are stored) or, if already stored, refreshed.
 */
cb_status cb_update(cb_ctx* ctx, const int32_t* tokens, int64_t row_stride, const int32_t* n_old,
                    const int32_t* n_new, void* stream);

/*
 * cb_update for long runs of new tokens (Section 3.3: the dynamic table is initialised with a sliding window over the
 * prompt).  Same arguments, same resulting tables, clocks and counters as cb_update; the work of one sequence is spread
 * over many warps where that cannot change the result (no leader can be evicted during the run: leaders stored + windows
 * <= LC, and at least 64 windows), and done by one warp in order otherwise.  Runs of up to 8,192 windows take one launch,
 * whose blocks reduce a run in shared memory without regard to its order (batches of up to 1,024 sequences, under the reading
 * that re-inserting a stored follower refreshes it); where row_stride has room for longer ones, or for more windows than LC,
 * two more belong to the call (seven with scratch attached, see below).  CB_CNT_FOLLOWER_EVICTIONS counts the followers this call displaced from the lists; with
 * scratch attached, where a run is reduced, a follower that the run itself would have stored and displaced again is never stored and
 * so is not counted.
 */
cb_status cb_update_bulk(cb_ctx* ctx, const int32_t* tokens, int64_t row_stride, const int32_t* n_old,
                         const int32_t* n_new, void* stream);

/*
 * Scratch memory for the order-free reduction of longer runs by cb_update_bulk.  After a run in which no leader can be evicted, and under the
 * reading that re-inserting a stored follower refreshes it (the default), a leader's stamp is that of its last window and its
 * followers are the FC distinct ones touched last (Section 3.1: both lists are least-recently-used lists), whatever the
 * order of the windows.  With scratch attached, the sequences of a call whose runs qualify (as above), have more than 8,192
 * windows and fit the scratch, taken in batch order, are reduced in it: one thread per window, then one warp per distinct leader.  The resulting
 * tables and clocks are those of cb_update; which place a follower or an entry takes inside the table may differ, which no
 * call reports.
 *   cb_bulk_scratch_bytes    HOST out: bytes for calls whose qualifying runs hold up to max_windows windows in total
 *                            (about 84 to 164 bytes per window: two hash tables of the next power of two >= 2 * max_windows
 *                            slots); cfg->batch sizes a small per-sequence array.
 *   cb_bulk_scratch_attach   dev_scratch: DEVICE, 256-byte aligned, `bytes` long, owned by the caller and to be kept while
 *                            attached; its content need not be initialised and is overwritten by every cb_update_bulk call.
 *                            NULL detaches.  Calls on one context that use it must not overlap.
 * Errors: CB_ERR_INVALID_ARG (null, misaligned, too small for any table).
 */
cb_status cb_bulk_scratch_bytes(const cb_config* cfg, int64_t max_windows, size_t* bytes);
cb_status cb_bulk_scratch_attach(cb_ctx* ctx, void* dev_scratch, size_t bytes);

/*
 * Draft-tree growth (Section 3.2).
 *   tokens, row_stride  as in cb_update;  seq_len int32 [batch] = tokens valid per sequence
 * Node 0 is the last token of the sequence (the one token whose K/V is not cached yet).  Level 1
 * queries the table with the last LL tokens of the sequence; every later level queries, for each leaf
 * that ends a complete follower, the last LL tokens of sequence ++ path-to-leaf.  Followers are
 * attached most recently inserted first, each as a chain of FL nodes; growth is breadth first and stops
 * at max_nodes (level 1 at max_nodes - crt), at max_depth, or when no leaf has a follower.  A chain
 * that does not fit is cut short and not grown further.  Every issued query refreshes its leader.
 * Outputs (all device):
 *   tree_tokens, tree_parent, tree_depth  int32 [batch, max_nodes]   parent of node 0 is -1
 *   tree_mask   uint32 [batch, max_nodes, W], W = ceil(max_nodes / 32): bit j of row i is set iff
 *               node j is node i or an ancestor of it
 *   n_nodes     int32 [batch]
 * A sequence with seq_len < 1 gets n_nodes = 0; with fewer than LL tokens, the root only.
 */
cb_status cb_draft_tree(cb_ctx* ctx, const int32_t* tokens, int64_t row_stride, const int32_t* seq_len,
                        int32_t* tree_tokens, int32_t* tree_parent, int32_t* tree_depth,
                        uint32_t* tree_mask, int32_t* n_nodes, void* stream);

/*
 * cb_update followed by cb_draft_tree on the grown sequences, in one launch (Section 3.2: the table is brought up to
 * date with the newly accepted tokens before the next draft is made from it).  Same arguments, results, table state
 * and errors as cb_update(tokens, row_stride, n_old, n_new) followed by cb_draft_tree(tokens, row_stride, n_new, ...);
 * at small batch the step saves a kernel boundary.
 */
cb_status cb_update_draft_tree(cb_ctx* ctx, const int32_t* tokens, int64_t row_stride, const int32_t* n_old,
                               const int32_t* n_new, int32_t* tree_tokens, int32_t* tree_parent, int32_t* tree_depth,
                               uint32_t* tree_mask, int32_t* n_nodes, void* stream);

/*
 * Extra branches from another drafter (Conclusion: because the drafts form a tree, the predicted drafts of other
 * speculative-decoding methods can be inserted as additional branches).  Call it between cb_draft_tree and the
 * verification pass.
 *   branches    int32 [batch, n_branches, max_len]   each row a run of tokens continuing the sequence after its last token
 *   branch_len  int32 [batch, n_branches]            tokens valid in each row (<= 0: none)
 *   n_branches <= 64
 * The tree arrays are those cb_draft_tree wrote and are extended in place.  For every sequence with a root, the branches
 * are taken in order; each becomes a chain of new nodes below the root (node 0), cut where the tree would exceed max_nodes
 * or a node max_depth, and ended by a negative token.  Branches are not compared with nodes already present.  The mask
 * rows of the new nodes and n_nodes are updated.  The tables are not touched.
 */
cb_status cb_tree_add_branches(cb_ctx* ctx, const int32_t* branches, const int32_t* branch_len, int32_t n_branches,
                               int32_t max_len, int32_t* tree_tokens, int32_t* tree_parent, int32_t* tree_depth,
                               uint32_t* tree_mask, int32_t* n_nodes, void* stream);

/*
 * Tree-masked attention over the paged KV cache (Section 3.2, "tree attention": a token attends only
 * to its ancestors in the draft tree; the cached context is fully visible).
 * With T = max_nodes, Hq / Hkv = n_q_heads / n_kv_heads, D = head_dim, P = page_size:
 *   q            bf16 [batch, T, Hq, D]
 *   k_pool,v_pool bf16 [num_pages, P, Hkv, D]   cached keys / values, paged
 *   block_table  int32 [batch, max_pages]       page id of the j-th page of each sequence
 *   ctx_len      int32 [batch]                  cached tokens per sequence (<= max_pages * P)
 *   k_tree,v_tree bf16 [batch, T, Hkv, D]       keys / values of the tree tokens themselves
 *   tree_mask    uint32 [batch, T, W], n_nodes int32 [batch]   as written by cb_draft_tree: node 0 is in the masks of all nodes
 *   out          bf16 [batch, T, Hq, D]         rows >= n_nodes are written as zero
 *   lse          float [batch, Hq, T] or NULL   natural-log sum of exponentials per row (0 for padding)
 *   max_ctx      host upper bound on every ctx_len (0 = max_pages * P); sizes the grid and, with few units, names the page-table entry of
 *                each sequence that is read ahead of its length (the entry is used only if the length says it is the one wanted)
 *   scale        softmax scale; 0 selects 1/sqrt(D)
 * Row (b, i, h) = softmax_j(scale * q.k_j) v_j over j in {cached tokens of kv head h / (Hq/Hkv)}
 * U {tree nodes in mask row i}; fp32 accumulation and softmax, output rounded to bf16.
 * Equal calls give equal bits.  How a row's keys are split for the sum follows from ctx_len and n_nodes of the whole batch, so the last
 * bits of a sequence's rows may depend on the other sequences.
 * All base pointers must be 16-byte aligned.
 * Keys and values are fetched a tile at a time and what lies outside a row's key set is given probability 0, not skipped,
 * so everything a tile covers must be finite (0 x NaN would reach the output): all T rows of k_tree / v_tree of every
 * sequence, including rows >= n_nodes, and the slots of a sequence's last, partly filled page beyond ctx_len.  Pages past
 * the last one are never read.  Buffers from an allocator that does not clear them must be zeroed once.
 */
typedef struct {
    const void* q;
    const void* k_pool;
    const void* v_pool;
    const int32_t* block_table;
    const int32_t* ctx_len;
    const void* k_tree;
    const void* v_tree;
    const uint32_t* tree_mask;
    const int32_t* n_nodes;
    void* out;
    float* lse;
    int32_t max_pages;
    int32_t num_pages;
    int32_t max_ctx;
    float scale;
} cb_attn_args;

cb_status cb_tree_attn(cb_ctx* ctx, const cb_attn_args* args, void* stream);

/*
 * Greedy acceptance (Section 3.2: the forward pass yields one more token than the accepted draft
 * tokens, so a step emits between 1 and 1 + longest-branch tokens).
 *   tree_tokens, tree_parent, tree_depth, n_nodes   as written by cb_draft_tree
 *   logits        [batch, max_nodes, vocab] of logits_dtype (CB_DTYPE_F32 / CB_DTYPE_BF16), node rows
 *                 logits_row_stride elements apart (sequence stride = max_nodes * logits_row_stride);
 *                 finite values only.  target[i] = index of the first maximum of row i.
 *   target_ids_in int32 [batch, max_nodes]: targets given directly.  Exactly one of logits /
 *                 target_ids_in is non-NULL.
 * Node i > 0 is verified iff its parent is verified and tree_tokens[i] == target[parent]; the root is
 * verified.  The deepest verified node wins (lowest index among equally deep ones).  With m its depth:
 *   n_accept       int32 [batch]               = m
 *   accept_nodes   int32 [batch, max_depth]    the m nodes below the root on the winning path
 *   out_tokens     int32 [batch, max_depth+1]  their tokens followed by target[winner]  (m+1 tokens)
 *   target_ids_out int32 [batch, max_nodes] or NULL: the argmax of every valid row (-1 for padding)
 */
cb_status cb_accept(cb_ctx* ctx, const int32_t* tree_tokens, const int32_t* tree_parent,
                    const int32_t* tree_depth, const int32_t* n_nodes, const void* logits,
                    int32_t logits_dtype, int64_t logits_row_stride, const int32_t* target_ids_in,
                    int32_t* n_accept, int32_t* accept_nodes, int32_t* out_tokens,
                    int32_t* target_ids_out, void* stream);

/*
 * One step's acceptance and the next step's update and draft in one launch (Fig. 2: per sequence the three follow one
 * another — the emitted tokens extend the sequence, their windows go into the table, the next tree is drafted from it).
 * Same results, table state, counters and errors as
 *   cb_accept(tree_*, n_nodes, logits, ..., NULL, n_accept, accept_nodes, out_tokens, target_ids_out);
 *   tokens[b][seq_len[b] .. seq_len[b] + n_accept[b] + 1) = out_tokens[b][0 .. n_accept[b] + 1);   old = seq_len;   seq_len += n_accept + 1;
 *   cb_update(tokens, row_stride, old, seq_len);   cb_draft_tree(tokens, row_stride, seq_len, next_*);
 * At small batch the step saves two kernel boundaries.
 *   logits .. target_ids_out   as in cb_accept (logits only)
 *   tokens      int32 [batch, row_stride]  DEVICE, read and written: the emitted tokens are appended
 *   seq_len     int32 [batch]              DEVICE, read and written: tokens valid per sequence
 *   next_tokens, next_parent, next_depth, next_mask, next_n_nodes   the next tree, as written by cb_draft_tree; they may be the
 *               arrays of the verified tree (a sequence's acceptance has read them before its draft writes them)
 * A sequence whose history has no room for the emitted tokens (seq_len + n_accept + 1 > row_stride) keeps its length, nothing
 * is appended, the draft is made from the sequence as it is, and CB_ERR_INVALID_ARG is recorded in the device status.  A
 * sequence with an empty tree (n_nodes = 0) emits nothing.
 */
typedef struct cb_accept_draft_args {
    const void* logits;
    int32_t logits_dtype;
    int64_t logits_row_stride;
    const int32_t* tree_tokens;
    const int32_t* tree_parent;
    const int32_t* tree_depth;
    const int32_t* n_nodes;
    int32_t* n_accept;
    int32_t* accept_nodes;
    int32_t* out_tokens;
    int32_t* target_ids_out;
    int32_t* tokens;
    int64_t row_stride;
    int32_t* seq_len;
    int32_t* next_tokens;
    int32_t* next_parent;
    int32_t* next_depth;
    uint32_t* next_mask;
    int32_t* next_n_nodes;
} cb_accept_draft_args;

cb_status cb_accept_update_draft_tree(cb_ctx* ctx, const cb_accept_draft_args* args, void* stream);

/*
 * KV commit of the accepted path (Section 3.2: the draft tokens and the pending token are the tokens of the
 * verification pass that have no cached K/V; once a branch is accepted its tokens are ordinary context for the next
 * step).  For every sequence b with m = n_accept[b], the tree root (node 0) and the accepted nodes accept_nodes[b, 0..m),
 * in that order, become context tokens ctx_len[b] .. ctx_len[b] + m: their rows of k_tree / v_tree are copied into the
 * paged cache (page block_table[b, pos / P], slot pos % P) and ctx_len[b] grows by m + 1.  The bonus token of cb_accept
 * has no K/V yet: it is the next step's root.
 *   k_pool, v_pool  bf16 [num_pages, P, Hkv, D]   written
 *   block_table     int32 [batch, max_pages]      must already name pages for the new positions
 *   ctx_len         int32 [batch]                 read and updated in place
 *   k_tree, v_tree  bf16 [batch, T, Hkv, D]
 *   n_accept        int32 [batch], accept_nodes int32 [batch, max_depth]   as written by cb_accept
 * A sequence with ctx_len + m + 1 > max_pages * P is left untouched and CB_ERR_KV_FULL is recorded in the device status;
 * a node or page index outside its tensor is skipped and recorded as CB_ERR_INVALID_ARG.  Only enqueues work.
 */
typedef struct {
    void* k_pool;
    void* v_pool;
    const int32_t* block_table;
    int32_t* ctx_len;
    const void* k_tree;
    const void* v_tree;
    const int32_t* n_accept;
    const int32_t* accept_nodes;
    int32_t max_pages;
    int32_t num_pages;
} cb_kv_commit_args;

cb_status cb_kv_commit(cb_ctx* ctx, const cb_kv_commit_args* args, void* stream);

/*
 * Queries, keys and values as a model's projection leaves them, for cb_chunk_append and cb_tree_rope (the paper leaves the model's own
 * layers to the caller; these calls make what cb_chunk_attn and cb_tree_attn read).  Per head: an RMS norm of queries and keys, and the
 * rotation by position in the same pass.  With x one head of a row, D = head_dim, R = rotary_dim:
 *   y = x / sqrt(mean(x^2) + eps) * w                       (no norm where w is NULL)
 *   (y_a, y_b) -> (y_a c_i - y_b s_i, y_b c_i + y_a s_i)     for i < R / 2, with (a, b) = (i, i + R / 2), or (2i, 2i + 1) if interleaved;
 *                                                            c_i = rope[pos][i], s_i = rope[pos][R / 2 + i]; elements from R on stay
 * in fp32, rounded to bf16 once at the end.  Values are copied.
 *   q, k, v     bf16; head h of row r starts q_stride * r + h * D elements from the base (k, v alike), so that the three may be parts of
 *               one projected row
 *   q_norm, k_norm  bf16 [D] or NULL
 *   rope        float [rope_len, R], or NULL for no rotation
 * Base pointers are 16-byte aligned, strides multiples of 8, R a multiple of 16 and at most D, eps >= 0.
 */
typedef struct {
    const void* q;
    const void* k;
    const void* v;
    int64_t q_stride, k_stride, v_stride;
    const void* q_norm;
    const void* k_norm;
    float eps;
    const float* rope;
    int32_t rope_len, rotary_dim, interleaved;
} cb_qkv_rows;

/*
 * Appends a chunk of new tokens per sequence (a prompt, a part of one, or a single token) to the paged cache and makes their queries.
 * The chunks lie one behind the other: sequence b's are rows q_start[b] .. q_start[b + 1), and row q_start[b] + i is the token at
 * position ctx_len[b] + i.
 *   q_start     int32 [batch + 1]               non-decreasing, <= n_rows; a sequence without new tokens has an empty range
 *   ctx_len     int32 [batch]                   tokens cached before this chunk; only read, so that every layer of a model can be given
 *                                               the same lengths (the caller adds the chunk lengths after the last one)
 *   block_table int32 [batch, max_pages]        must already name pages for the new positions
 *   q_out       bf16 [n_rows, Hq, D]            may be q itself where q_stride = Hq * D
 *   k_pool, v_pool  bf16 [num_pages, P, Hkv, D] written at the new positions only
 * Rows that belong to no sequence (before q_start[0], from q_start[batch] on) are left as they were.  A sequence whose pages cannot
 * hold the new tokens is left alone (no row of it is written) and CB_ERR_KV_FULL is recorded in the device status; one whose range is not
 * inside [0, n_rows] or whose ctx_len is negative, and a row whose position the rope table does not have or whose page lies outside the
 * pool, are left alone and CB_ERR_INVALID_ARG recorded.
 */
typedef struct {
    cb_qkv_rows rows;
    const int32_t* q_start;
    const int32_t* ctx_len;
    const int32_t* block_table;
    int32_t n_rows;
    int32_t max_pages;
    int32_t num_pages;
    void* q_out;
    void* k_pool;
    void* v_pool;
} cb_chunk_append_args;

cb_status cb_chunk_append(cb_ctx* ctx, const cb_chunk_append_args* args, void* stream);

/*
 * The same for the nodes of a draft tree before their verification pass: row b * T + i is node i of sequence b, at position
 * ctx_len[b] + tree_depth[b][i] (T = max_nodes; the root is the first token that is not cached).
 *   tree_depth int32 [batch, T], n_nodes int32 [batch]   as written by cb_draft_tree;  ctx_len int32 [batch]
 *   q_out bf16 [batch, T, Hq, D]; k_out, v_out bf16 [batch, T, Hkv, D]   the tensors that cb_tree_attn and cb_kv_commit read; each may be
 *              its input where that is laid out the same way
 * Rows from n_nodes on are written as zero (cb_tree_attn wants them finite).  A node whose position the rope table does not have is
 * written as zero and CB_ERR_INVALID_ARG recorded.
 */
typedef struct {
    cb_qkv_rows rows;
    const int32_t* tree_depth;
    const int32_t* n_nodes;
    const int32_t* ctx_len;
    void* q_out;
    void* k_out;
    void* v_out;
} cb_tree_rope_args;

cb_status cb_tree_rope(cb_ctx* ctx, const cb_tree_rope_args* args, void* stream);

/*
 * Causal attention of each sequence's chunk of new tokens over its paged cache, the chunk's own keys and values included
 * (cb_chunk_append has put them there): row q_start[b] + i attends to cached positions 0 .. ctx_len[b] + i.
 *   q            bf16 [n_rows, Hq, D]
 *   k_pool, v_pool, block_table   as in cb_tree_attn;  q_start, ctx_len   as in cb_chunk_append
 *   out          bf16 [n_rows, Hq, D]
 *   lse          float [n_rows, Hq] or NULL     natural-log sum of exponentials per row
 *   max_chunk    host upper bound on every chunk length (0 = n_rows); with chunks of few tokens it decides how the work is split
 *   max_ctx      host upper bound on every ctx_len + chunk length (0 = max_pages * P)
 *   scale        softmax scale, positive and finite; 0 selects 1/sqrt(D)
 * fp32 accumulation and softmax, output rounded to bf16; equal calls give equal bits, as in cb_tree_attn.
 * Rows that belong to no sequence are left as they were.  A sequence whose cached and new tokens exceed max_pages * P, or max_ctx, is
 * left alone and CB_ERR_KV_FULL recorded; one whose range is not inside [0, n_rows], or longer than max_chunk, or whose ctx_len is
 * negative, is left alone and CB_ERR_INVALID_ARG recorded.  A page outside the pool reads as zeros.
 * Slots of the last, partly filled page beyond the sequence's tokens may hold anything; the tokens' own keys and values must be finite.
 * out must not be q.  Base pointers are 16-byte aligned.
 */
typedef struct {
    const void* q;
    const void* k_pool;
    const void* v_pool;
    const int32_t* block_table;
    const int32_t* q_start;
    const int32_t* ctx_len;
    void* out;
    float* lse;
    int32_t n_rows;
    int32_t max_pages;
    int32_t num_pages;
    int32_t max_chunk;
    int32_t max_ctx;
    float scale;
} cb_chunk_attn_args;

cb_status cb_chunk_attn(cb_ctx* ctx, const cb_chunk_attn_args* args, void* stream);

/*
 * Block tables made on the GPU.  The pages of a pool that no sequence holds lie on a stack; one call gives pages to the sequences that
 * grow and takes them back from those that shrink, so that a step's lengths never have to reach the host.
 *   want_len    int32 [batch]               tokens that each sequence is to have room for (0: it is finished)
 *   block_table int32 [batch, max_pages]    read and written: the first held[b] entries of row b are its pages
 *   held        int32 [batch]               read and written: pages of each sequence
 *   free_pages  int32 [num_pages]           read and written: the stack, its top at n_free[0] - 1
 *   n_free      int32 [1]                   read and written
 * With t = ceil(want_len / P), a sequence that holds more than t pages gives the ones behind the first t back, one that holds fewer is given
 * t - held.  What is there to give is, in this order: the pages given back in this call, by sequence and place, then the stack from its
 * top; the sequences that grow take from it one after the other, and what is left of the pages given back is pushed so that the first of them
 * is at the top.  (A call that grows some sequences is undone by one that shrinks them to where they were.)  Where the needs up to and with
 * a growing sequence exceed what there is, it is left alone, and so are the growing ones behind it; CB_ERR_KV_FULL is recorded.  So is a
 * sequence whose t exceeds max_pages.  A sequence with a negative length, or whose held is not in 0 .. max_pages, is left alone and
 * CB_ERR_INVALID_ARG recorded; a stack whose n_free is not in 0 .. num_pages, or that the pages given back would overfill, leaves everything as it
 * is and records the same.  Entries behind a row's pages and behind the top of the stack are not touched.  batch <= CB_MAX_ASSIGN,
 * num_pages < 2^30.
 */
enum { CB_MAX_ASSIGN = 16384 };
cb_status cb_pages_assign(cb_ctx* ctx, const int32_t* want_len, int32_t* block_table, int32_t max_pages, int32_t* held, int32_t* free_pages,
                          int32_t num_pages, int32_t* n_free, void* stream);

/*
 * Where the rows of a packed batch go (as in cb_chunk_append): row q_start[b] + i is the token at position ctx_len[b] + i of sequence b.
 *   slots      int64 [n_rows]   block_table[b][pos / P] * P + pos % P, the row of the pool seen as [num_pages * P, ...]
 *   positions  int32 [n_rows], seqs int32 [n_rows]
 * Rows that belong to no sequence are -1 in all three, as are those of a sequence whose range is not inside [0, n_rows] or whose ctx_len is
 * negative (CB_ERR_INVALID_ARG recorded) or whose pages cannot hold its tokens (CB_ERR_KV_FULL).  A row whose page lies outside the pool
 * has slot -1 and CB_ERR_INVALID_ARG is recorded.
 */
typedef struct {
    const int32_t* q_start;
    const int32_t* ctx_len;
    const int32_t* block_table;
    int32_t max_pages;
    int32_t num_pages;
    int32_t n_rows;
    int64_t* slots;
    int32_t* positions;
    int32_t* seqs;
} cb_slot_map_args;

cb_status cb_slot_map(cb_ctx* ctx, const cb_slot_map_args* args, void* stream);

/*
 * Attention over the parts of a long context that matter: the context is cut into blocks of `block` tokens (16, 32, 64 or 128), every block has a
 * summary (its mean key, in 8 bits), and per sequence and kv head the queries of a chunk or of a tree choose n_select blocks by it.
 *
 * cb_block_summary: the summaries of the blocks that new tokens touch, after their keys are in the pages (cb_chunk_append, cb_kv_commit).  For
 * every block that holds one of the positions from_len[b] .. to_len[b] - 1 of sequence b, over its tokens below to_len[b], m = sum of a head's keys / tokens:
 *   k_scale = max |m| / 127,   k_mean[d] = m[d] * 127 / max(max |m|, 1e-30) rounded to the nearest whole number (half way: to the even one)
 * each operation in 64 bits.  The sum is exact there, and so independent of any order of addition, unless the exponents of a channel's keys lie more than 38
 * apart; then too it is taken in one order whatever the call: equal keys give equal bits.  They are stored with the block's first page.
 *   k_pool   bf16 [num_pages, P, Hkv, D];  block_table int32 [batch, max_pages];  from_len, to_len int32 [batch]
 *   k_mean   int8 [num_pages, Hkv, D], k_scale float [num_pages, Hkv]     other pages' rows are left as they were
 * A head whose mean is not finite gets k_scale = +inf and zeros, which cb_block_select puts before all others.  A sequence with
 * from_len >= to_len has none; one with from_len < 0 is left alone and CB_ERR_INVALID_ARG recorded, one with to_len > max_pages * P CB_ERR_KV_FULL; a
 * block with a page outside the pool is left alone and CB_ERR_INVALID_ARG recorded.  batch <= CB_MAX_ASSIGN, batch * ceil(max_pages * P / block) < 2^30.
 * Sequences that share pages (a common prefix) share their blocks' summaries: a block whose first page they share has to be the same in all of its pages and tokens.
 */
typedef struct {
    const void* k_pool;
    const int32_t* block_table;
    const int32_t* from_len;
    const int32_t* to_len;
    int8_t* k_mean;
    float* k_scale;
    int32_t max_pages;
    int32_t num_pages;
    int32_t block;
} cb_block_summary_args;

cb_status cb_block_summary(cb_ctx* ctx, const cb_block_summary_args* args, void* stream);

/*
 * cb_block_select: which blocks of its cached tokens each sequence's new rows attend to, one list per kv head.  The rows are a chunk's
 * (q_start given: rows q_start[b] .. q_start[b + 1) of q [n_rows, Hq, D]) or a tree's (n_nodes given: the first n_nodes[b] of q [batch, T, Hq, D]).
 * All query heads of the kv head and all rows vote: with a = max |q| over them (at least 1e-30) and r = 127 / a,
 *   q8 = q * r rounded to a whole number (fp32),   score_j = float(max over rows and heads of sum_d q8[d] k_mean_j[d]) * k_scale_j
 * Sums of whole numbers: the choice depends on no order of addition.  Of the nb = ceil(ctx_len / block) blocks the n_first first and the
 * n_last newest ones are always chosen, the others by falling score, equal scores by rising number, until there are n_select; a score that is not a
 * number comes before all others.
 *   ctx_len  int32 [batch]   cached tokens before the chunk or the tree
 *   blocks   int32 [batch, Hkv, n_select]   by rising number; -1 behind the last where nb < n_select; all -1 where there are no rows
 *   n_first >= 0, n_last >= 1, n_first + n_last <= n_select <= CB_MAX_SELECT
 *   max_chunk  host upper bound on a chunk's rows (0 = n_rows; more than 20,000,000 may be turned away as if it were above the bound), max_ctx on
 *              every ctx_len (0 = max_pages * P); max_ctx / block <= 16,384.  max_chunk is worth giving: with at most 16 queries a kv head, max_chunk
 *              * Hq / Hkv, units are taken by a kernel for few queries (64 single tokens: a third of the time).  One long chunk takes all
 *              sequences of its call to the other kernel.
 * A sequence whose rows or ctx_len are out of their bounds (q_start's range, n_nodes, max_chunk; negative ctx_len: CB_ERR_INVALID_ARG; ctx_len > max_ctx:
 * CB_ERR_KV_FULL) gets -1 throughout.  A block whose first page lies outside the pool scores as if k_scale were 0, CB_ERR_INVALID_ARG recorded.  Queries
 * are finite.
 */
enum { CB_MAX_SELECT = 1024 };
typedef struct {
    const void* q;
    const int32_t* q_start;
    const int32_t* n_nodes;
    const int8_t* k_mean;
    const float* k_scale;
    const int32_t* block_table;
    const int32_t* ctx_len;
    int32_t* blocks;
    int32_t n_rows;
    int32_t max_pages;
    int32_t num_pages;
    int32_t block;
    int32_t n_select, n_first, n_last;
    int32_t max_chunk;
    int32_t max_ctx;
} cb_block_select_args;

cb_status cb_block_select(cb_ctx* ctx, const cb_block_select_args* args, void* stream);

/*
 * Attention over the selected blocks.
 *   cb_block_attn       cb_chunk_attn in which row q_start[b] + i sees, of the ctx_len[b] cached tokens, only those in its kv head's blocks, and
 *                       the chunk's own tokens up to its own
 *   cb_block_tree_attn  cb_tree_attn in which the cached context is that of the kv head's blocks; masks of any form (a row that sees no token and no
 *                       node is zero, its lse too)
 * max_chunk decides between two kernels here too: with max_chunk * Hq / Hkv <= 16 a call of single tokens takes 17 to 50% less time than as a call of chunks, which
 * it is taken for without that bound.
 * Arguments, outputs, errors and alignment are those of the dense calls (max_ctx bounds what it bounds there: a chunk's cached and new tokens, a tree's
 * cached ones).  A tree whose n_nodes is not in 0 .. T or whose ctx_len is negative (CB_ERR_INVALID_ARG recorded), or whose ctx_len exceeds max_ctx or
 * max_pages * P (CB_ERR_KV_FULL), gets zeros as if it had no nodes; without nodes its ctx_len is not looked at.  blocks int32 [batch, Hkv,
 * n_select] is as cb_block_select leaves it for the same ctx_len and block: with nb = ceil(ctx_len / block) > n_select a list names n_select
 * blocks below nb, the newest one last; with fewer its first nb entries are 0 .. nb - 1.  Other lists give rows of no meaning; a block that does
 * not exist, or a page outside the pool, reads as zeros.
 */
cb_status cb_block_attn(cb_ctx* ctx, const cb_chunk_attn_args* args, const int32_t* blocks, int32_t block, int32_t n_select, void* stream);
cb_status cb_block_tree_attn(cb_ctx* ctx, const cb_attn_args* args, const int32_t* blocks, int32_t block, int32_t n_select, void* stream);

/*
 * How likely tokens were: for each of n_out rows of logits x over vocab tokens, with Z = sum_v exp(x_v),
 *   logprobs[i]  = x_t - log Z              t = tokens[i]
 *   entropy[i]   = log Z - sum_v p_v x_v    p = exp(x) / Z
 *   top_ids[i], top_logprobs[i]             the top_k largest x_v (equal ones by rising id) and their x_v - log Z, largest first
 * fp32 throughout.  Logits are finite or -inf (a forbidden token: probability 0, no part of the entropy); a row with a NaN or +inf, or
 * without a finite logit, gives NaN; its alternatives are ids all the same, -1 where only NaNs are left.
 *   logits        [n_rows, vocab] of logits_dtype, rows logits_row_stride elements apart
 *   rows          int32 [n_out]: the row of logits of each output, or NULL for row i (n_out <= n_rows)
 *   tokens        int32 [n_out], or NULL: logprobs is then not written
 *   logprobs, entropy  float [n_out], each or NULL
 *   top_ids       int32 [n_out, top_k], top_logprobs float [n_out, top_k]; top_k 0..CB_MAX_TOP; with fewer than top_k tokens in the vocabulary the
 *                 rest is -1 and -inf
 * An output with a negative token, or a negative row, is padding: its row is not read, logprobs and entropy are 0, top_ids -1,
 * top_logprobs 0.  A token >= vocab or a row >= n_rows is treated the same way and CB_ERR_INVALID_ARG recorded.
 *
 * cb_accept_logprobs: the same for the tokens that cb_accept emitted, from the logits it was given.  Output (b, j) is for
 * out_tokens[b][j], whose row is that of node 0 for j = 0 and of accept_nodes[b][j - 1] behind it; the places behind the bonus token
 * (out_tokens -1) are padding.  Outputs have leading dimensions [batch, max_depth + 1]; logits are [batch, max_nodes, vocab].
 */
enum { CB_MAX_TOP = 32 };
typedef struct {
    const void* logits;
    int32_t logits_dtype;
    int64_t logits_row_stride;
    int32_t n_rows;
    int32_t n_out;
    const int32_t* rows;
    const int32_t* tokens;
    int32_t top_k;
    float* logprobs;
    float* entropy;
    int32_t* top_ids;
    float* top_logprobs;
} cb_logprobs_args;

cb_status cb_logprobs(cb_ctx* ctx, const cb_logprobs_args* args, void* stream);
/* args->n_rows, n_out, rows and tokens are not read. */
cb_status cb_accept_logprobs(cb_ctx* ctx, const int32_t* accept_nodes, const int32_t* out_tokens, const cb_logprobs_args* args, void* stream);

/*
 * Frozen table (Section 3.3): a second, read-only table built offline from the most frequent leader-follower pairs of a
 * corpus.  A step drafts from the dynamic table first and then lets the frozen table add branches while the tree is below
 * its size cap; insertions never reach it.
 *
 * A frozen table is one device buffer owned by the caller, of cb_frozen_bytes() bytes, 256-byte aligned, shared by every
 * sequence and every context that attaches it, and only read by the step calls.  LL and FL must equal the context's;
 * LC (1..2^20) and FC (1..128) are its own.
 *
 *   cb_frozen_load    fills the buffer from HOST arrays: leaders int32 [n_leaders, LL], n_followers int32 [n_leaders]
 *                     (1..FC each), followers int32 [n_leaders, FC, FL], each leader's followers most frequent first,
 *                     leaders most frequent first.  Synchronises the device.
 *   cb_frozen_dump    the reverse, into HOST arrays sized for LC leaders (any may be NULL; unused follower places -1):
 *                     leaders by falling corpus count, equal counts by rising tokens.  Synchronises the device.
 *   cb_frozen_attach  makes cb_draft_tree of this context run the second pass; dev_table = NULL detaches.  Host call, no
 *                     device work; order it against draft calls in flight yourself.
 *
 * With a frozen table attached, cb_draft_tree continues after the dynamic pass while the tree has fewer than max_nodes
 * nodes: it visits, first in first out, every node that can carry a follower list (the root and the last node of every
 * complete follower, in creation order; the ends of the complete followers the frozen pass adds join the queue), looks
 * the node's key up in the frozen table and attaches the stored followers, most frequent first, under the same rules as
 * the dynamic pass (a query at the root only while fewer than max(1, max_nodes - crt) nodes exist, any other while fewer
 * than max_nodes; max_depth; a follower that does not fit is cut short).  Frozen followers are not compared with the
 * branches already present.  Frozen queries touch no recency and are counted in CB_CNT_FROZEN_QUERIES / _HITS.
 *
 * Offline construction (Section 4: from a corpus sample, the LC most frequent n-grams of length LL become the leaders,
 * and each leader keeps the FC most frequent n-grams of length FL that follow it).
 *   cb_frozen_build   counts on the GPU.  dev_corpus int32 [n_tokens] (device, ids >= 0, one token stream,
 *                     n_tokens <= 2^30); an occurrence is counted where LL + FL tokens are available, so every leader
 *                     has at least one follower; equal counts are ordered by the tokens, smallest first.  dev_scratch:
 *                     cb_frozen_build_bytes() bytes of device memory, 256-byte aligned, free again after the call.
 *                     Overwrites dev_table.  Enqueues on `stream` and waits for it; returns CB_ERR_INVALID_ARG if a
 *                     negative token was met (its windows are left out).
 */
typedef struct {
    int32_t LL, FL, LC, FC;
} cb_frozen_config;

cb_status cb_frozen_bytes(const cb_frozen_config* cfg, size_t* bytes);
cb_status cb_frozen_load(const cb_frozen_config* cfg, void* dev_table, size_t bytes, int32_t n_leaders,
                         const int32_t* leaders, const int32_t* n_followers, const int32_t* followers);
cb_status cb_frozen_dump(const cb_frozen_config* cfg, const void* dev_table, size_t bytes, int32_t* n_leaders,
                         int32_t* leaders, int32_t* n_followers, int32_t* followers);
cb_status cb_frozen_attach(cb_ctx* ctx, const cb_frozen_config* cfg, const void* dev_table, size_t bytes);
cb_status cb_frozen_build_bytes(const cb_frozen_config* cfg, int64_t n_tokens, size_t* scratch_bytes);
cb_status cb_frozen_build(const cb_frozen_config* cfg, const int32_t* dev_corpus, int64_t n_tokens, void* dev_table,
                          size_t table_bytes, void* dev_scratch, size_t scratch_bytes, void* stream);

/*
 * cb_accept_static — cb_accept (logits form) for callers that must not allocate device memory.
 * (The paper has no counterpart; this is a packaging variant of the call above.)
 *
 * Who needs it: code that runs where cudaMalloc is off limits — inside a framework's memory pool whose
 * owner forbids side allocations, in a plugin that is handed buffers but no allocator, or under a
 * memory budget that is fixed before the library is loaded.  Such a caller cannot provide the workspace
 * cb_create wants, so this entry point needs no context at all: the scratch that the arg-max reduction
 * uses (one packed maximum per logits row and one arrival counter per sequence) lives in a fixed array
 * that is part of the library image.  Every GPU that loads the library carries that array
 * (CB_STATIC_MAX_ROWS * 8 + CB_STATIC_MAX_BATCH * 4 bytes = 68 KiB) until the process exits.
 *
 * Shape arguments replace the context: batch, max_nodes (1..128), max_depth (>= 0), vocab (>= 1).
 * All other arguments, the result and the tie rules are exactly those of cb_accept with logits given;
 * target_ids_out may be NULL.
 *
 * Limits: batch <= CB_STATIC_MAX_BATCH and batch * max_nodes <= CB_STATIC_MAX_ROWS; anything larger
 * returns CB_ERR_STATIC_LIMIT and enqueues nothing.
 *
 * The call never allocates or frees (no cudaMalloc / cudaFree, no allocating library routine).  The first
 * call on each device looks up the array's device address once, with that device current; make that
 * first call outside any stream capture.  Before each launch the part of the array in use is cleared
 * on `stream`.  All calls on a device share the one array: two calls that may overlap on the GPU
 * (different streams without an ordering between them) race on it and give wrong results; order them.
 */
enum { CB_STATIC_MAX_BATCH = 1024, CB_STATIC_MAX_ROWS = 8192 };
cb_status cb_accept_static(int32_t batch, int32_t max_nodes, int32_t max_depth, int32_t vocab,
                           const int32_t* tree_tokens, const int32_t* tree_parent, const int32_t* tree_depth,
                           const int32_t* n_nodes, const void* logits, int32_t logits_dtype,
                           int64_t logits_row_stride, int32_t* n_accept, int32_t* accept_nodes,
                           int32_t* out_tokens, int32_t* target_ids_out, void* stream);

/*
 * Canonical view of one sequence's table, for checkpointing and for comparing table contents:
 * leaders least recently used first, each leader's followers least recently inserted first.
 * HOST buffers: leaders int32 [LC, LL], n_followers int32 [LC], followers int32 [LC, FC, FL]
 * (unused follower slots -1); any of them may be NULL.  *n_leaders receives the count.  Synchronises.
 */
cb_status cb_table_dump(cb_ctx* ctx, int32_t seq, int32_t* n_leaders, int32_t* leaders,
                        int32_t* n_followers, int32_t* followers);

/* Replaces one sequence's table by the given canonical content (same HOST layouts as cb_table_dump;
 * recency = position). Synchronises. */
cb_status cb_table_load(cb_ctx* ctx, int32_t seq, int32_t n_leaders, const int32_t* leaders,
                        const int32_t* n_followers, const int32_t* followers);

/*
 * Reads (and clears) the device status word and copies the counters to the HOST array `counters`
 * (CB_NUM_COUNTERS entries, may be NULL).  Synchronises.
 */
enum {
    CB_CNT_INSERTS = 0,
    CB_CNT_LEADER_EVICTIONS = 1,
    CB_CNT_FOLLOWER_EVICTIONS = 2,
    CB_CNT_QUERIES = 3,
    CB_CNT_QUERY_HITS = 4,
    CB_CNT_MAX_PROBE = 5,
    CB_CNT_FROZEN_QUERIES = 6,
    CB_CNT_FROZEN_HITS = 7,
    CB_NUM_COUNTERS = 8
};
cb_status cb_poll_status(cb_ctx* ctx, cb_status* device_status, uint64_t* counters);

/*
 * 1 if this library is the checking build (compiled with -DCB_DEBUG), else 0.  No counterpart in the paper: the checking
 * build is the stand-in for a memory checker.  In it every table slot, entry id, page id and node index that a kernel takes
 * from memory is range-checked before use (a value out of range records CB_ERR_INVALID_ARG in the device status and the
 * access is skipped; nothing traps), and every workspace region is followed by 256 guard bytes that cb_poll_status verifies
 * (CB_ERR_CANARY if one changed).  cb_workspace_bytes is larger in that build.  Results are identical to the regular build.
 */
int cb_debug_build(void);

/* Kernels launched by this library since the process started (host-side count). */
uint64_t cb_launch_count(void);

const char* cb_status_str(cb_status s);

#ifdef __cplusplus
}
#endif
#endif /* CACHEBACK_H_ */
