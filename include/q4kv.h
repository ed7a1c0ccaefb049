/*
 * q4kv.h -- C ABI of libq4kv: batched attention over many agents' paged, 4-bit
 * group-quantized KV caches on one AMD MI355X (gfx950), plus the Q4 pack/unpack
 * codec used when a cache is saved or restored.
 *
 * Conventions that hold for every entry point
 *   - "device" pointers are GPU global memory owned by the caller (for example the
 *     storage of a torch tensor).  The library allocates no device memory and keeps
 *     no state between calls.  "host" pointers are ordinary process memory.
 *   - Calls only enqueue work on `hip_stream` (a hipStream_t passed as void*, NULL =
 *     the default stream) and return without synchronising.
 *   - Return value: Q4KV_OK (0) or a negative q4kv_status.  Argument errors are found
 *     on the host before anything is launched; q4kv_last_error() then gives a message
 *     (thread-local, valid until the same thread's next failing call).
 *   - binary16 values travel as uint16_t bit patterns.  Inputs must be finite.
 *   - Calls that overlap in time on different streams are safe as long as their
 *     output and workspace buffers do not overlap.
 *
 * The Q4 format (Sec. 3.2 "Q4 Quantization Pipeline" of the paper; arithmetic fixed
 * by the project brief where the paper defers to its framework): a row of `dim`
 * elements is cut into groups of 64 consecutive elements along head_dim.  Per group:
 *     bias  = min x                          stored as binary16 (exact)
 *     scale = (max x - min x) / 15           computed in binary32, stored as binary16 (RNE)
 *     code  = clamp(rint((x - min) / scale_stored), 0, 15)   binary32 division, ties to even;
 *             all codes 0 when scale_stored == 0
 * Element d of a row lives in 32-bit word d/8, bits 4*(d%8) .. 4*(d%8)+3.
 * The paper stores scale and bias as bfloat16 for one model family and as binary16 for another (Sec. 3.1, Sec. 3.2,
 * appendix "safetensors Q4 Format").  Q4KV_PARAMS_BF16 selects the bfloat16 form: the same formula with both
 * parameters rounded to bfloat16 (nearest even) and the codes taken against the STORED parameters,
 *     code = clamp(rint((x - bias_stored) / scale_stored), 0, 15),
 * so a reader needs nothing but the stored values.  The stored bias is then in general not the minimum itself:
 * |x - x_hat| <= scale_stored/2 + |bias_stored - min| + 15 |scale_stored - scale|.  Parameters must stay inside the
 * binary16 range (they do for binary16 data).
 * Bytes per row: dim/2 (codes) + 2*dim/64 (scale) + 2*dim/64 (bias), i.e. K+V of a
 * layer take h*d*n*(1 + 8/64) bytes, the paper's count.
 */
#ifndef Q4KV_H
#define Q4KV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    Q4KV_OK = 0,
    Q4KV_EINVAL = -1,     /* null / misaligned pointer, negative count, bad layer range */
    Q4KV_ESHAPE = -2,     /* unsupported dims: dim % 64, q_heads % kv_heads, head widths, group/block size */
    Q4KV_ERANGE = -3,     /* max_seq_len exceeds what the block table can address, or chunk_len its limit */
    Q4KV_EWORKSPACE = -4, /* workspace too small or missing */
    Q4KV_EHIP = -5,       /* the HIP runtime refused a launch */
    Q4KV_ENOSPACE = -6    /* the block pool has too few free blocks (nothing was changed) */
} q4kv_status;

/* Type of the stored scale and bias values (both 16 bits wide, so layouts and byte counts do not change). */
typedef enum {
    Q4KV_PARAMS_F16 = 0,  /* IEEE binary16 */
    Q4KV_PARAMS_BF16 = 1  /* bfloat16 */
} q4kv_param_format;

/* Shape descriptor of one model's cache: the paper's ModelCacheSpec (Sec. 3.1, and
 * Sec. 3.6 for v_dim != k_dim).  The library reads nothing model-specific beyond it. */
typedef struct {
    int32_t num_layers;
    int32_t num_q_heads;
    int32_t num_kv_heads;   /* divides num_q_heads; query head h reads KV head h / (num_q_heads/num_kv_heads) */
    int32_t k_dim;          /* multiple of 64 */
    int32_t v_dim;          /* multiple of 64 */
    int32_t v_aliases_k;    /* 1: a token's V row is the first v_dim elements of its K row (one shared
                               latent per token); the V pool argument must then be NULL */
    int32_t block_tokens;   /* 256, the paper's block size (Sec. 3.1) */
    int32_t group_size;     /* 64 */
    int32_t param_format;   /* q4kv_param_format of every pool used with this spec */
} q4kv_spec;

/* One paged Q4 pool (K or V) for all layers, device memory, row-major:
 *   codes [num_layers][num_blocks][num_kv_heads][block_tokens][dim/8]   uint32
 *   scale [num_layers][num_blocks][num_kv_heads][block_tokens][dim/64]  binary16 (or bfloat16) bits
 *   bias  same shape as scale
 * All three base pointers must be 16-byte aligned.  A block id indexes the second axis;
 * an agent owns the blocks its block-table row lists (Sec. 3.1, per-agent isolation). */
typedef struct {
    uint32_t *codes;
    uint16_t *scale;
    uint16_t *bias;
    int32_t num_blocks;
} q4kv_pool;

/* Sec. 3.2, the "save" half of the codec.  Quantize `rows` rows of `dim` binary16 values.
 *   x      device, [rows][dim], 16-byte aligned
 *   codes  device out, [rows][dim/8]; scale, bias device out, [rows][dim/64]
 * Bit-exact with the definition above.  rows == 0 is a no-op.  dim % 64 != 0 -> Q4KV_ESHAPE. */
int q4kv_quantize(const uint16_t *x, int64_t rows, int32_t dim, uint32_t *codes, uint16_t *scale, uint16_t *bias,
                  void *hip_stream);

/* Sec. 3.2 / Sec. 4.4 (the dequantization cost on restore): x_hat = code*scale + bias in
 * binary32, rounded to binary16.  Arguments mirror q4kv_quantize; x is the device output. */
int q4kv_dequantize(const uint32_t *codes, const uint16_t *scale, const uint16_t *bias, int64_t rows, int32_t dim,
                    uint16_t *x, void *hip_stream);

/* The two calls above with the type of scale and bias chosen by `param_format` (a q4kv_param_format; anything
 * else -> Q4KV_EINVAL).  Q4KV_PARAMS_F16 is exactly q4kv_quantize / q4kv_dequantize. */
int q4kv_quantize_fmt(const uint16_t *x, int64_t rows, int32_t dim, int32_t param_format, uint32_t *codes,
                      uint16_t *scale, uint16_t *bias, void *hip_stream);
int q4kv_dequantize_fmt(const uint32_t *codes, const uint16_t *scale, const uint16_t *bias, int64_t rows, int32_t dim,
                        int32_t param_format, uint16_t *x, void *hip_stream);

/* Sec. 3.4, first half of update_and_fetch: quantize new K/V rows and store them behind
 * each agent's cached tokens.
 *   k_new, v_new    device, [layer_end-layer_begin][num_agents][chunk_len][num_kv_heads][dim] binary16
 *                   (v_new and v must be NULL when spec->v_aliases_k)
 *   block_table     device int32 [num_agents][max_blocks]; entry i of a row is the physical block that
 *                   holds tokens 256*i .. 256*i+255 of that agent; it must already list the blocks the
 *                   new tokens fall into
 *   seq_len_before  device int32 [num_agents], tokens cached before this call
 * Token seq_len_before[a]+c of agent a receives chunk row c.  A token whose table slot is beyond
 * max_blocks or whose block id is outside the pool is skipped (nothing is written for it).
 * chunk_len > Q4KV_MAX_CHUNK_LEN -> Q4KV_ERANGE (the kernel places rows with quotients that are exact up
 * to there); longer chunks are appended in pieces. */
#define Q4KV_MAX_CHUNK_LEN (1 << 20)
int q4kv_append(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const uint16_t *k_new,
                const uint16_t *v_new, const int32_t *block_table, int32_t max_blocks,
                const int32_t *seq_len_before, int32_t num_agents, int32_t chunk_len, int32_t layer_begin,
                int32_t layer_end, void *hip_stream);

/* q4kv_append for a batch in which every agent brings a number of tokens of its own: rows of new tokens one behind the other, and
 * the place of each in the pools (a slot map, as q4kv_resize_tables writes it) instead of a chunk length.
 *   k_new, v_new  device, [layers of the call][num_tokens] token rows, each token's heads contiguous ([num_kv_heads][dim]);
 *                 *_stride elements from one token row to the next, so that they may be parts of one fused projection.  Strides
 *                 are multiples of 8 and no smaller than a row, pointers 16-byte aligned.  v_new must be NULL when
 *                 spec->v_aliases_k.  in_format: 0 binary16, 1 bfloat16 (of both): a bfloat16 value is rounded once to binary16,
 *                 and must be inside its range
 *   slot          device int32 [num_tokens]: block * 256 + place in the block, the same on every layer.  A token whose slot is
 *                 outside [0, 256 * num_blocks) is skipped (-1 for the tokens that fill a batch up): its rows may hold anything, and
 *                 may be read.  Tokens with one slot are not put in order: each word of codes, scale and bias there is one of
 *                 theirs, but a group's codes may stand beside another token's scale, so the slot's value means nothing
 * The cache gets the bits that q4kv_append makes of the same rows.  num_tokens > Q4KV_MAX_CHUNK_LEN, pools of 2^23 blocks and
 * more and calls of 2^31 groups and more on a layer -> Q4KV_ERANGE. */
int q4kv_append_slots(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const void *k_new, const void *v_new,
                      int32_t in_format, int64_t k_stride, int64_t v_stride, const int32_t *slot, int32_t num_tokens,
                      int32_t layer_begin, int32_t layer_end, void *hip_stream);

/* What a model does to the heads of Q and K between a layer's projections and the cache (Sec. 3.6 names the models).  For
 * every head row x of k_dim elements:
 *   norm      elements i < norm_dim become x_i * weight[i] / sqrt(mean of x_j^2 over j < norm_dim + eps); the others stay.
 *             q_weight and k_weight are device binary32 [layers of the call][norm_dim]; NULL: no norm on Q (on K)
 *   rotation  of the elements rot_begin .. rot_begin + rot_dim - 1, after the norm: pair (y_i, y_j) of a token at position p
 *             becomes (y_i c - y_j s, y_j c + y_i s) with c = cos_table[p][n], s = sin_table[p][n] (device binary32
 *             [table_len][rot_dim / 2]) for the n-th pair: n and n + rot_dim / 2 inside the span, or with `neighbours` != 0
 *             2n and 2n + 1.  rot_dim == 0: none, the tables are not read.
 * norm_dim and rot_begin are multiples of 8, rot_dim of 16, both spans lie inside k_dim and may overlap; weights and tables
 * are 16-byte aligned.  Results are those of binary64 arithmetic rounded once to binary16 (but for one within 2^-48 of
 * |y_i c| + |y_j s| of a rounding border); where the elements under the norm are all zero they stay zeros whatever eps is. */
typedef struct {
    const float *q_weight, *k_weight;
    const float *cos_table, *sin_table;
    int32_t norm_dim; /* 0 where neither Q nor K is normed */
    float eps;        /* >= 0 */
    int32_t rot_begin, rot_dim, neighbours, table_len;
} q4kv_head_form;

/* q4kv_append behind that: one pass from the projections of new tokens to their queries and cache rows.
 *   q, k_new, v_new  device, [layers of the call][num_agents][chunk_len] token rows, each token's heads contiguous
 *                    ([num_q_heads][k_dim], [num_kv_heads][k_dim], [num_kv_heads][v_dim]); *_stride elements from one token
 *                    row to the next, so that the three may be parts of one fused projection.  Strides are multiples of 8
 *                    and no smaller than a row, pointers 16-byte aligned.  v_new must be NULL when spec->v_aliases_k.
 *                    in_format: 0 binary16, 1 bfloat16 (a q4kv_param_format, of all three); values must be finite and, as
 *                    prepared, inside the binary16 range
 *   q_out            device out, binary16 [layers][num_agents][chunk_len][num_q_heads][k_dim], 16-byte aligned: what
 *                    q4kv_batched_attention takes as q.  May not overlap the inputs.
 *   positions        device int32 [num_agents][chunk_len], or NULL: seq_len_before[a] + c for token c of agent a
 * V rows are quantized as they are.  Block tables, seq_len_before and skipped tokens as for q4kv_append (a token that finds no
 * slot still gets its query); with a rotation, a token whose position is outside [0, table_len) is skipped whole: neither its
 * query nor its rows are written.  The cache gets the bits that q4kv_append makes of the same prepared rows.  Rows of more than
 * 1,024 elements -> Q4KV_ESHAPE. */
int q4kv_norm_rope_append(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const q4kv_head_form *form,
                          const void *q, const void *k_new, const void *v_new, int32_t in_format, int64_t q_stride,
                          int64_t k_stride, int64_t v_stride, uint16_t *q_out, const int32_t *block_table,
                          int32_t max_blocks, const int32_t *seq_len_before, const int32_t *positions,
                          int32_t num_agents, int32_t chunk_len, int32_t layer_begin, int32_t layer_end,
                          void *hip_stream);

/* Sec. 3.4, second half of update_and_fetch, and Sec. 3.6 (GQA grouping, causal chunk masks):
 * out = softmax(sm_scale * q K_hat^T) V_hat per agent, layer and query head, directly on the Q4
 * pools (nothing is dequantized to memory).
 *   q            device, [layer_end-layer_begin][num_agents][q_len][num_q_heads][k_dim] binary16.  With q_len > 1 and on a
 *                shared latent no 64 elements of a group may sum up to more than 65504 (plain decode has no such bound)
 *   out          device out, same leading shape, v_dim wide, binary16
 *   seq_len      device int32 [num_agents]: keys visible to the LAST query row of each agent, the
 *                appended chunk included; row r sees the first seq_len[a] - (q_len-1-r) tokens
 *                (q_len == 1: decode).  A row with no visible key yields zeros.
 *   max_seq_len  host upper bound of seq_len[]; it sizes the launch.  seq_len values above it are
 *                clamped to it on the device.  max_seq_len > max_blocks*256 -> Q4KV_ERANGE.
 *   window       <= 0: global attention.  > 0: row at position p also requires t > p - window
 *                (sliding-window layers, Sec. 3.6).
 *   split_tokens smallest token range handed to one wavefront (multiple of 256), 0 = library picks.  The
 *                tokens of all (layer, KV head, agent) units are dealt out evenly over a fixed set of
 *                wavefronts; this is the floor of a wavefront's share and bounds the partial results kept
 *                per query head.  Must equal the value given to q4kv_attention_workspace_bytes.  With 0 the share may
 *                become smaller than q4kv_default_split_tokens says where the lengths are far below max_seq_len.
 *   workspace    device scratch of at least q4kv_attention_workspace_bytes(...) bytes, 16-byte aligned;
 *                contents before and after the call are unspecified.  (Of the size told for split_tokens == 0 a call on a
 *                shared latent needs only the part that it is told for q4kv_default_split_tokens, and deals out coarser
 *                ranges with less than the whole: a workspace sized for a larger batch serves the smaller ones.)  With q_len > 1 it is optional: a call whose
 *                workspace_bytes is exactly what q4kv_attention_workspace_bytes says may use it to spread few or ragged
 *                agents over the whole chip.  Its contents (a decode plan, say) are then lost, and calls that overlap in
 *                time need one each.  With any other workspace_bytes (a decode call's workspace) or NULL the call
 *                runs as well and does not touch the workspace.
 * Per-agent isolation (Sec. 3.1): nothing an agent's table row does not list up to seq_len ever enters its result,
 * and the kernels read no block the row does not list: slots past seq_len that a tile's loads touch lie in the
 * agent's own last block, and a block id outside [0, num_blocks) is skipped (its tokens count as masked; the loads
 * go to the agent's own first block instead, or to block 0 if that id is outside the pool too, and are discarded).
 * Outputs are run-to-run bit-identical for identical arguments.  The order in which an agent's tokens are summed
 * follows from the sizes of the call (agents, layers, max_seq_len, window), from the lengths of all its agents, and from the
 * workspace (with q_len > 1 whether it has its own, on a shared latent whether it has the whole size), so an agent's bits
 * may differ between calls that batch it differently or beside an agent that has grown. */
int q4kv_batched_attention(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const uint16_t *q,
                           uint16_t *out, const int32_t *block_table, int32_t max_blocks, const int32_t *seq_len,
                           int32_t num_agents, int32_t q_len, int32_t max_seq_len, float sm_scale, int32_t window,
                           int32_t split_tokens, int32_t layer_begin, int32_t layer_end, void *workspace,
                           size_t workspace_bytes, void *hip_stream);

/* Sec. 3.6 (models that interleave global and sliding-window layers): q4kv_batched_attention with one window per
 * layer of the call instead of a single one.
 *   window_per_layer  HOST int32 [layer_end - layer_begin], read before the call returns; entry i belongs to layer
 *                     layer_begin + i; <= 0: global attention on that layer.
 * At most 128 layers per call (more -> Q4KV_EINVAL; split the layer range).  Everything else, the workspace size
 * included, is as for q4kv_batched_attention, but that q_len > 1 with more than one layer makes no use of a workspace.
 * On decode the tokens a window hides are never read. */
int q4kv_batched_attention_windows(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const uint16_t *q,
                                   uint16_t *out, const int32_t *block_table, int32_t max_blocks,
                                   const int32_t *seq_len, int32_t num_agents, int32_t q_len, int32_t max_seq_len,
                                   float sm_scale, const int32_t *window_per_layer, int32_t split_tokens,
                                   int32_t layer_begin, int32_t layer_end, void *workspace, size_t workspace_bytes,
                                   void *hip_stream);

/* The decode step of a forward pass is one call per layer (the next layer's queries depend on this layer's output),
 * all with the same lengths, and then the small kernel that turns seq_len[] into the launch's work plan is a tenth of
 * every call.  These two entry points take it out of the loop (Sec. 3.4, the decode loop of a batch):
 *   q4kv_decode_plan                writes the plan for calls of `num_layers_in_call` layers with these lengths, this
 *                                   window (one for all layers, <= 0: global) and this split_tokens into `workspace`
 *   q4kv_batched_attention_planned  q4kv_batched_attention with q_len == 1 on a workspace prepared that way: no
 *                                   seq_len argument (the plan holds the lengths, clamped to max_seq_len), one kernel
 * Every argument the two share must be the same in both calls (the layer range may differ from call to call, its
 * length may not), and seq_len[] must not be relied on to have changed in between: the planned call attends to the
 * lengths the plan was made from.  A workspace may be used for any number of planned calls on one stream, one after
 * the other; when the lengths change (every decode step), or another call has used the workspace, plan again (a call
 * with q_len > 1 uses one of its own size only, see `workspace` above).  A workspace prepared for other arguments
 * makes the planned call do nothing (it is detected on the device; `out` is left as it was); so does a plan for a shared
 * latent that was given the whole size told for split_tokens == 0 when the planned call is given less.  Shapes, workspace size,
 * error codes and results (bit-identical to q4kv_batched_attention with the same arguments) as described there. */
int q4kv_decode_plan(const q4kv_spec *spec, const int32_t *seq_len, int32_t num_agents, int32_t max_seq_len,
                     int32_t window, int32_t split_tokens, int32_t num_layers_in_call, void *workspace,
                     size_t workspace_bytes, void *hip_stream);
int q4kv_batched_attention_planned(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const uint16_t *q,
                                   uint16_t *out, const int32_t *block_table, int32_t max_blocks, int32_t num_agents,
                                   int32_t max_seq_len, float sm_scale, int32_t window, int32_t split_tokens,
                                   int32_t layer_begin, int32_t layer_end, void *workspace, size_t workspace_bytes,
                                   void *hip_stream);

/* Decode attention (q_len == 1) of agents that share prefixes: q4kv_batched_attention on global layers, with the tokens that
 * a group of agents has in common read once for up to 32 of its query rows on a KV head, 48 with 64-wide heads (Sec. 3.4, the decode
 * loop of a batch; q4kv_block_pool_fork makes such agents).  With ten agents of two query heads per KV head behind a common prompt of
 * 8,192 tokens the cache that a step reads is a seventh.  The plain calls read shared blocks correctly too, once per agent: next to
 * q4kv_batched_attention_planned, one layer a call, this one is the faster from four agents and about 4,096 shared tokens on, and
 * the slower below 1,024.
 *   group_begin  device int32 [num_groups + 1]: group g is agents group_begin[g] .. group_begin[g + 1] - 1; ascending.  Agents
 *                outside all groups share nothing.  Bounds that fall are read as the largest one in front of them, and bounds
 *                outside [0, num_agents] as the nearest in it.
 *   prefix_len   device int32 [num_groups]: the first prefix_len[g] tokens are the same for all agents of group g.  They are read
 *                through the block-table row of the group's FIRST agent, which must list them, in whole 64-token tiles (what is
 *                left of the last one is read through every agent's own row, as are its further tokens), and no further than
 *                max_seq_len.  A row sees the first seq_len[a] tokens as ever, also where that is less than prefix_len.
 *   num_groups   0: nobody shares anything, the two arrays may be NULL.  No more than num_agents
 *   workspace    device scratch of at least q4kv_shared_prefix_workspace_bytes(...) bytes, 16-byte aligned; contents before and
 *                after the call are unspecified.  Calls that overlap in time need one each.
 * All other arguments, block ids outside the pool (masked; the loads go to block 0 and are discarded), rows that see no token (zeros)
 * and run-to-run identical bits as for q4kv_batched_attention; the order of a row's sum is another one, so the bits are in general
 * not that call's.  Q4KV_ERANGE: more than 512 agents; 2^24 (layer, agent, query head) rows or 2^21 (layer, KV head) pairs and more;
 * tiles of 64 tokens (layers * KV heads * (agents + row tiles) * max_seq_len / 64) close to 2^31 and more.  Head shapes: k_dim == v_dim of 64, 128 or 256, or 192 and 128; at most 16 query heads per KV
 * head; no shared latent (Q4KV_ESHAPE). */
int q4kv_shared_prefix_attention(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const uint16_t *q,
                                 uint16_t *out, const int32_t *block_table, int32_t max_blocks, const int32_t *seq_len,
                                 int32_t num_agents, const int32_t *group_begin, const int32_t *prefix_len,
                                 int32_t num_groups, int32_t max_seq_len, float sm_scale, int32_t layer_begin,
                                 int32_t layer_end, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Bytes of workspace q4kv_shared_prefix_attention needs for these arguments, whatever the groups.  0 on bad arguments.  A row (layer,
 * agent, query head) may leave a record of v_dim + 2 binary32 values per range of 128 tokens and more, but no more than
 * 1,024 / (layers * KV heads) + 4 (256 compute units): 12 MB for one layer of ten agents of 9,000 tokens with 32 query and 8 KV
 * heads, 128-wide, 72 MB for two of 32 behind 16,384, 1.1 GB for one of 512 agents and 131,072. */
size_t q4kv_shared_prefix_workspace_bytes(const q4kv_spec *spec, int32_t num_agents, int32_t max_seq_len,
                                          int32_t num_layers_in_call);

/* For callers that cannot allocate device memory or have none to hand over -- code recording a HIP graph, tight
 * serving loops that call once per layer, harnesses that forbid hipMalloc: q4kv_batched_attention with the decode
 * path's workspace (tile plan and partial results) taken from a fixed array of Q4KV_STATIC_SCRATCH_BYTES bytes that
 * the library's code object holds on every GPU it is loaded on, from the first use of the library on that GPU until
 * the process ends.  No workspace arguments; everything else, q and out (caller-owned device memory) included, is as
 * for q4kv_batched_attention, and the results are bit-identical to that call with the same split_tokens -- with
 * q_len > 1, to that call without its optional workspace (a chunk call takes nothing from the array).
 *   - The call allocates nothing and frees nothing, on the device or through any library.  The first call on a
 *     device looks the array's address up once (with that device current, as for every call); make that first call
 *     outside a graph capture.
 *   - q4kv_attention_workspace_bytes(...) > Q4KV_STATIC_SCRATCH_BYTES -> Q4KV_EWORKSPACE, nothing is launched: pass
 *     fewer layers per call or a larger split_tokens.  One layer of every benchmark configuration fits, in 11 MB at most, but
 *     that of five 32,768-token agents on a shared latent, which needs 21.2 MB (10.7 with split_tokens 512).
 *   - Every call on a GPU shares that GPU's one array, which keeps the last call's contents (nothing in it has to
 *     start at zero that the call's own first kernel does not write): calls that overlap in time on one GPU, on
 *     different streams or from different threads, race on it and are not allowed.  Calls on one stream are ordered
 *     by the stream. */
#define Q4KV_STATIC_SCRATCH_BYTES (16u << 20)
int q4kv_batched_attention_static(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const uint16_t *q,
                                  uint16_t *out, const int32_t *block_table, int32_t max_blocks,
                                  const int32_t *seq_len, int32_t num_agents, int32_t q_len, int32_t max_seq_len,
                                  float sm_scale, int32_t window, int32_t split_tokens, int32_t layer_begin,
                                  int32_t layer_end, void *hip_stream);

/* Bytes of workspace q4kv_batched_attention needs for these arguments.  0 on bad arguments (q4kv_last_error() then
 * holds a message).  For q_len > 1 the bytes with which the call may share its work out evenly over the compute units
 * (it runs without them too, one workgroup per row tile): up to 136 MB on a GPU of 256 compute units, whatever the
 * lengths; 0 where it never does.  No q_len == 1 call is told that number, and a chunk call goes by it (see `workspace`
 * above): pass it as workspace_bytes even if the buffer is larger. */
size_t q4kv_attention_workspace_bytes(const q4kv_spec *spec, int32_t num_agents, int32_t q_len, int32_t max_seq_len,
                                      int32_t split_tokens, int32_t num_layers_in_call);

/* The split size the library would pick for split_tokens == 0 (0 on bad arguments). */
int32_t q4kv_default_split_tokens(const q4kv_spec *spec, int32_t num_agents, int32_t q_len, int32_t max_seq_len,
                                  int32_t num_layers_in_call);

/* Sec. 3.2 closed form: Q4 bytes (K and V, all layers) of `tokens` cached tokens:
 * layers * kv_heads * (k_dim + v_dim) * tokens * (1/2 + 4/64); v_dim counts 0 when V aliases K.
 * Negative on bad arguments. */
int64_t q4kv_cache_bytes(const q4kv_spec *spec, int64_t tokens);

/* Saving and restoring an agent's cache (Sec. 3.1 block pool; Sec. 3.2 "Q4 at rest"; appendix "safetensors Q4
 * Format": one tensor per layer, block and array, Q4 on disk exactly as in memory, so that a restore is a copy and
 * no prefill).  A block image is the contiguous form of `num_blocks` listed blocks of every layer of the spec:
 *   for layer l = 0 .. num_layers-1, for i = 0 .. num_blocks-1 (block block_ids[i]):
 *     K codes uint32 [kv_heads][256][k_dim/8], K scale binary16 [kv_heads][256][k_dim/64], K bias (same shape),
 *     V codes, V scale, V bias likewise with v_dim (absent when v_aliases_k)
 * i.e. the pool's own bytes of that (layer, block), array after array.  q4kv_block_image_bytes gives its size
 * (0 on bad arguments).  q4kv_export_blocks gathers pool -> image, q4kv_import_blocks scatters image -> pool
 * (into whatever blocks block_ids names now: a restored agent need not get its old blocks back).
 *   block_ids  device, int32 [num_blocks]; an id outside [0, pool.num_blocks) is skipped (its records are left
 *              untouched on export, nothing is written on import)
 *   image      device (or pinned host memory the GPU can address), 16-byte aligned, at least image_bytes long
 *              With the image in host memory the launch is kept small (the host link, not the chip, is the
 *              limit), so that it can run beside a decode step on another stream.
 * Enqueue on hip_stream, allocate nothing, never synchronise.  Q4KV_EWORKSPACE when image_bytes is too small. */
size_t q4kv_block_image_bytes(const q4kv_spec *spec, int32_t num_blocks);
int q4kv_export_blocks(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const int32_t *block_ids,
                       int32_t num_blocks, void *image, size_t image_bytes, void *hip_stream);
int q4kv_import_blocks(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const int32_t *block_ids,
                       int32_t num_blocks, const void *image, size_t image_bytes, void *hip_stream);

/* Copies blocks inside the pools: block dst_ids[i] of every layer, K and V, codes and parameters, becomes a copy of block
 * src_ids[i].  What a fork's last block and the moves of a compaction need (q4kv_block_pool_fork, _truncate, _compact hand out
 * the pairs), with nothing in between.
 *   src_ids, dst_ids  device, int32 [num_pairs]; a pair with an id outside [0, pool.num_blocks) or of one id twice is skipped.
 *                     A block may be the source of any number of pairs; one that is the destination of two pairs, or of one
 *                     and the source of another, holds afterwards a mixture of their bytes.
 * Enqueues on hip_stream, allocates nothing.  At most 65,535 layers. */
int q4kv_copy_blocks(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const int32_t *src_ids,
                     const int32_t *dst_ids, int32_t num_pairs, void *hip_stream);

/* Block tables that live on the GPU.  q4kv_block_pool_* (below) keeps who owns which block on the host; a serving loop or a beam
 * search that never waits for the GPU keeps the same in device memory, and the calls behind this struct work on it in stream
 * order.  A row is an agent (a request, a beam); it lists the ceil(seq_len / 256) blocks of its tokens in token order.
 *   block_table  device int32 [num_agents][max_blocks], what every attention and append call takes; entries behind a row's blocks
 *                mean nothing (an entry that a call takes away becomes -1)
 *   seq_len      device int32 [num_agents], tokens cached (read as 0 below 0, as 256 * max_blocks above that)
 *   refs         device int32 [num_blocks]: rows that list the block, of this table or of any other with these pools; 0: free.  A
 *                program that keeps blocks for itself (a prompt's image, say) counts itself in
 *   refused      device int32 [1] or NULL: set by every call to the number of rows that did not get what they asked for
 * A block that several rows list is full of tokens that they all have; the block that a row ends in, if it is not full, is its
 * own.  The calls here keep it so, as far as blocks last.  Free blocks are handed out lowest id first, to rows in order: results are the same on
 * every run.  At most Q4KV_MAX_TABLE_ROWS rows and 2^23 - 1 blocks, 2^31 - 1 tokens a row (Q4KV_ERANGE); calls on one table, or on tables
 * with the same refs, must not overlap in time.  An entry outside [0, num_blocks) is carried along and counted nowhere.  Tables of no
 * rows need none of the first three arrays (NULL). */
#define Q4KV_MAX_TABLE_ROWS 2048
typedef struct {
    int32_t *block_table, *seq_len, *refs, *refused;
    int32_t num_agents, max_blocks, num_blocks;
} q4kv_tables;

/* The agents' lengths become new_len[], and their tables with them: what q4kv_block_pool_reserve, _truncate and _release do for one
 * agent on the host, for all of them at once.
 *   new_len       device int32 [num_agents]: tokens from now on.  0 gives all blocks back, a negative one leaves the row as it is
 * Rows that get shorter free their blocks first, so that the same call can hand them out.  Free blocks go to rows in order.  Rows
 * that get longer are served up to the first whose blocks are not there, or whose tokens do not fit the map; that one and
 * the growing rows behind it are left as they were (and counted in refused) and take no blocks, as is a row whose new length its table
 * cannot list.
 * A slot map of the tokens that rows got longer by, agent after agent, for q4kv_append_slots:
 *   max_tokens    places in it; 0: none wanted, and no bound on the tokens
 *   token_begin   device out, int32 [num_agents + 1]: first token of each agent, and their number
 *   slot, token_agent, position   device out, int32 [max_tokens]: block * 256 + place, row, and place in the agent's text of each
 *                 token; -1 behind the last one.  token_agent and position may be NULL
 * With spec and pools (spec NULL: none), a row that goes on, or is cut, or stays, inside a block that others list as well gets a copy
 * of that block's first tokens, every layer, and goes on in that (of rows that all end there, and with nobody else listing it, the
 * lowest keeps the block; but it gets a copy too where it grows and a row that has more tokens there gets none).  Where no block is
 * left for the copy, a row that is cut loses what it has of the shared block: its seq_len becomes the multiple of 256 below, and it
 * counts as refused; a row that stays, or was refused, keeps it, shared as it is.  Without pools all but that lowest row lose what
 * they have of a shared block that they are cut inside, and a row that goes on is taken to end in a block of its own.
 *   workspace     device scratch of q4kv_tables_workspace_bytes(num_agents) bytes, 16-byte aligned, contents unspecified; not
 *                 needed (NULL) without pools
 * Allocates nothing, never synchronises. */
int q4kv_resize_tables(const q4kv_tables *tables, const int32_t *new_len, int32_t max_tokens, int32_t *token_begin, int32_t *slot,
                       int32_t *token_agent, int32_t *position, const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v,
                       void *workspace, size_t workspace_bytes, void *hip_stream);

/* What a beam search does to the cache once it has chosen: row i of the tables becomes what row parent[i] was before the call
 * (parent: device int32 [num_agents]; a row whose parent is outside [0, num_agents) becomes empty).  Blocks are listed by one more row
 * or by one less; nothing is copied but the last block, if it is not full, of a row with several children: the lowest child goes
 * on in it, the others get free blocks with a copy of its seq_len % 256 tokens, every layer, K and V (what is in the other slots
 * of such a block is not touched).  A child for which no block is left keeps the full blocks only: its seq_len becomes the
 * multiple of 256 below, and it counts in refused.  With a parent listed for rows that were empty, this is the fork of an
 * agent, or of a prompt into its beams.  Workspace as above, needed always. */
int q4kv_beam_reorder(const q4kv_spec *spec, const q4kv_pool *k, const q4kv_pool *v, const q4kv_tables *tables, const int32_t *parent,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

/* Bytes of workspace of the two calls above.  0 on bad arguments. */
size_t q4kv_tables_workspace_bytes(int32_t num_agents);

/* The choice of a beam search's step.  Rows of logits are grouped (a request's beams); every row's continuations have the totals
 *     score[row] + x[token] - log(sum over tokens of exp x)
 * and of all continuations of a group's rows the num_out largest come out, largest first, equal ones in the order of row, then
 * logit (the larger first), then token.
 *   logits      device [num_agents][vocab], logits_format 0 binary16, 1 bfloat16 (a q4kv_param_format), 2 binary32; row_stride
 *               elements from one row to the next, any alignment that the type has.  -inf: a banned token, never chosen.  NaN
 *               counts as -inf, +inf as the largest finite binary32 number
 *   score       device binary32 [num_agents]; a row of score -inf (or NaN) has no continuation and is not read: the state before the
 *               first step is one beam of score 0 beside dead ones
 *   end_token   device int32 [num_agents] or NULL.  Not negative: the row is finished, its logits are not read, and its one
 *               continuation is that token, at the row's own score
 *   group_begin device int32 [num_groups + 1], as for q4kv_shared_prefix_attention: group g is rows group_begin[g] ..
 *               group_begin[g + 1] - 1 (bounds outside [0, num_agents] are read as the nearest in it; of bounds that fall the group
 *               is empty)
 *   num_out     1 .. Q4KV_MAX_BEAM_OUT for every group, whatever its rows.  With the group's number of rows, parent[] is what
 *               q4kv_beam_reorder takes
 *   parent, token, total   device out, int32, int32 and binary32 [num_groups][num_out]; where a group has no more continuations:
 *               -1, -1, -inf
 *   workspace   device scratch of q4kv_beam_select_workspace_bytes(...) bytes, 16-byte aligned, contents unspecified; calls
 *               that overlap in time need one each
 * Totals are formed and compared in binary64, from logarithms that are within (1.1 ln(vocab) + 18) 2^-23 of the true ones, and rounded
 * once to binary32 on their way out; the order within a row is that of its logits, exactly.  Run-to-run identical.  Rows times spans of
 * vocab (of 2,048 tokens at least) at most 2^26 - 4, at most 2^22 - 1 groups, vocab at most 2^30 (Q4KV_ERANGE).  Allocates nothing, never
 * synchronises. */
#define Q4KV_MAX_BEAM_OUT 64
int q4kv_beam_select(const void *logits, int32_t logits_format, int64_t row_stride, int32_t vocab, int32_t num_agents, const float *score,
                     const int32_t *end_token, const int32_t *group_begin, int32_t num_groups, int32_t num_out, int32_t *parent,
                     int32_t *token, float *total, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Bytes of workspace of q4kv_beam_select on the current device.  0 on bad arguments. */
size_t q4kv_beam_select_workspace_bytes(int32_t logits_format, int32_t vocab, int32_t num_agents, int32_t num_out);

/* Sec. 3.1 "Block Pool with Per-Agent Isolation", host side: which 256-token block of the device pools belongs to
 * which agent.  Pure bookkeeping in HOST memory (no device call): a block id is either free or in exactly one agent's
 * list, so two agents can never share or overwrite a block (the paper's namespace isolation) -- unless the caller forks an
 * agent, whose full blocks parent and child then both list and neither writes to (below); the list order is the
 * token order, i.e. a row of the block table the attention calls read.  Eviction is the caller's sequence
 * lru_victim -> q4kv_export_blocks -> (file) -> release; a restore is reserve -> q4kv_import_blocks into whatever blocks
 * were free.  Agent ids are caller-chosen non-negative numbers.  Every call locks the pool (thread-safe).
 *   create        a pool over block ids 0 .. num_blocks-1, all free; NULL on a bad argument or out of memory
 *   reserve       make the agent own ceil(tokens/256) blocks: blocks it has stay (in place and order), missing ones
 *                 come from the free list, lowest id first; an unknown agent is created; the agent becomes the most
 *                 recently used.  Never shrinks.  Returns the number of blocks owned, Q4KV_ENOSPACE when the free
 *                 list is too short (nothing changed), Q4KV_EINVAL on a negative id or token count
 *   release       free all blocks of the agent and forget it; returns the number freed, Q4KV_EINVAL if unknown
 *   blocks        copy the agent's block ids in token order into ids[0 .. cap) (host); returns how many it owns
 *   table_row     the same as a block-table row: ids, then `fill` up to max_blocks; Q4KV_ERANGE if it owns more
 *   touch         mark the agent most recently used;  pin(1): never a victim while it is in a running batch
 *   lru_victim    the unpinned agent with at least one block that was used least recently, or -1
 *   free_blocks   length of the free list;  owner: the agent id that owns a block (the smallest of those that share it), or -1
 * Agents that share a prefix:
 *   fork          a new agent `child` that has the first `tokens` cached tokens of `parent`: it lists the parent's
 *                 tokens / 256 full blocks too and, where tokens are left over, a free block of its own that must become a
 *                 copy of the parent's: *copy_from and *copy_to (host) get that pair for q4kv_copy_blocks, or -1.  Returns the
 *                 number of blocks the child lists; Q4KV_EINVAL if the child is known already or the parent is not,
 *                 Q4KV_ERANGE if the parent has not that many blocks, Q4KV_ENOSPACE (nothing changed)
 *   truncate      the agent keeps its first `tokens` tokens: blocks behind them are freed (shared ones when nobody else lists
 *                 them).  A block that stays in part and is shared is replaced by a free one, with its pair in *copy_from and
 *                 *copy_to (else -1).  Returns the number of blocks it still lists; errors as for fork
 *   compact       moves blocks to lower ids until the blocks in use are the lowest ones, but for those of pinned agents, which
 *                 stay; lists change at once, and the pairs in copy_from[], copy_to[] (host, [cap]) are to be given to ONE call of
 *                 q4kv_copy_blocks (no block is in both) before any of the blocks is used.  Returns the number of pairs;
 *                 Q4KV_ERANGE when there are more than cap (nothing changed).  cap == 0: only counts
 *   shares        agents that list a block (0: free)
 * release frees a shared block with the last agent that lists it, and returns the number of blocks freed.  A block is shared
 * only while it is full of tokens that all its agents have, so appending behind one's tokens never writes into it. */
typedef struct q4kv_block_pool q4kv_block_pool;
q4kv_block_pool *q4kv_block_pool_create(int32_t num_blocks);
void q4kv_block_pool_destroy(q4kv_block_pool *pool);
int32_t q4kv_block_pool_reserve(q4kv_block_pool *pool, int64_t agent_id, int64_t tokens);
int32_t q4kv_block_pool_release(q4kv_block_pool *pool, int64_t agent_id);
int32_t q4kv_block_pool_blocks(q4kv_block_pool *pool, int64_t agent_id, int32_t *ids, int32_t cap);
int32_t q4kv_block_pool_table_row(q4kv_block_pool *pool, int64_t agent_id, int32_t *row, int32_t max_blocks, int32_t fill);
int32_t q4kv_block_pool_touch(q4kv_block_pool *pool, int64_t agent_id);
int32_t q4kv_block_pool_pin(q4kv_block_pool *pool, int64_t agent_id, int32_t pinned);
int64_t q4kv_block_pool_lru_victim(q4kv_block_pool *pool);
int32_t q4kv_block_pool_free_blocks(q4kv_block_pool *pool);
int64_t q4kv_block_pool_owner(q4kv_block_pool *pool, int32_t block_id);
int32_t q4kv_block_pool_fork(q4kv_block_pool *pool, int64_t parent_id, int64_t child_id, int64_t tokens, int32_t *copy_from,
                             int32_t *copy_to);
int32_t q4kv_block_pool_truncate(q4kv_block_pool *pool, int64_t agent_id, int64_t tokens, int32_t *copy_from,
                                 int32_t *copy_to);
int32_t q4kv_block_pool_compact(q4kv_block_pool *pool, int32_t *copy_from, int32_t *copy_to, int32_t cap);
int32_t q4kv_block_pool_shares(q4kv_block_pool *pool, int32_t block_id);

/* Measurement helper, no part of the method: a kernel that only reads.  Reads the first
 * floor(bytes / 16384) * 16384 bytes of the device buffer `src` (16-byte aligned) exactly once, in the launch
 * shape and with the load width of the decode kernel, and writes nothing except, possibly, the one device word
 * `sink` (its value means nothing).  Timing it gives the read bandwidth the memory system sustains, against which
 * the benchmark quotes the decode kernel next to the published peak.  Enqueues on hip_stream; no allocation, no
 * synchronisation.  Fewer than 16,384 bytes: nothing happens.  Q4KV_EINVAL on a NULL or misaligned pointer. */
int q4kv_read_probe(const void *src, size_t bytes, uint32_t *sink, void *hip_stream);

/* Message of this thread's most recent failing call ("" if none). */
const char *q4kv_last_error(void);

/* Library version, major*10000 + minor*100 + patch. */
int q4kv_version(void);

#ifdef __cplusplus
}
#endif
#endif /* Q4KV_H */
