/*
 * hs_kernel.h - single-kernel entry points of the stage engine.
 *
 * These run one of the engine's HIP kernels on caller-owned device buffers,
 * exactly as the stage forward pass launches it. They exist so that each
 * kernel can be checked against a reference and timed on its own; serving
 * goes through hs.h. The cache operators at the end are operators of their own, for
 * servers that call the attention themselves. All pointers are device pointers owned by the caller;
 * `stream` is a hipStream_t (NULL = the null stream). Work is asynchronous,
 * except where an entry says that it waits.
 * Shapes the kernel does not support return HS_EINVAL before any launch.
 */
#ifndef HS_KERNEL_H
#define HS_KERNEL_H

#include <stdint.h>

#include "hs.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Y[m][n] = epilogue(sum_k X[m][k] W[n][k]) with fp32 accumulation. X is
 * bf16 row-major with row stride ldx (elements); W is the [N][K] matrix in
 * the tiled matrix format of hs.h (hs_pack_tiled). epi: 0 store bf16; 1 add
 * the bf16 residual R (row stride ldr; may alias Y); 2 SwiGLU on gate/up rows
 * interleaved in groups of 16, Y has N/2 columns; 3 store float32. Requires
 * K % 8 == 0, N % 16 == 0 (N % 32 for SwiGLU), 16-byte aligned X, W, Y; if
 * K % 64 != 0, ldx must be at least K rounded up to 64 and the extra columns
 * of X zero. This is the projection arithmetic of every decoder layer (QKV,
 * O, gate/up, down) and of the LM head. From 17 rows on, shapes with few
 * output tiles split their k range over workgroups; the partial sums go through
 * workspaces that the library allocates once per device (on the first call of
 * their size) and keeps until the process ends. Calls of up to 16 rows use none;
 * those of 17 to 64 rows share one of 8 MiB + 1 KiB and may come from any stream
 * or thread (the library orders the launches that split; a captured launch is
 * ordered by the caller); calls of more than 64 rows share one of 32 MiB +
 * 1 KiB and must not run concurrently on one device. Results are
 * deterministic: the same inputs give the same bits on every call. */
hs_status hs_k_gemm(const void* X, int64_t ldx, const void* W, void* Y, int64_t ldy,
                    const void* R, int64_t ldr, int32_t M, int32_t N, int32_t K, int32_t epi,
                    void* stream);

/* The same product with the RMSNorm of X's rows folded in (the norm of
 * section 2.1's decoder layer before attention and before the FFN):
 * Y = epilogue(rmsnorm(X) W^T) with rmsnorm(x) = x / sqrt(mean(x^2) + eps) * g,
 * g a bf16 [K] gain. X holds the raw rows; every activation is multiplied
 * by the gain and rounded to bf16 on the way into the product, and each
 * output row is scaled by its 1 / RMS in float32 afterwards. For decode
 * batches: requires 1 <= M <= 16 and K % 64 == 0 (HS_EINVAL otherwise);
 * other arguments and epilogues as hs_k_gemm. */
hs_status hs_k_gemm_rmsnorm(const void* X, int64_t ldx, const void* g, float eps, const void* W,
                            void* Y, int64_t ldy, const void* R, int64_t ldr, int32_t M,
                            int32_t N, int32_t K, int32_t epi, void* stream);

/* Causal grouped-query attention over packed sequences (the attention of the
 * prefill pass). qkv: bf16 [T][(n_heads + 2 n_kv_heads) head_dim] holding
 * post-RoPE q, k, v per token; out: bf16 [T][n_heads head_dim]; cu_seqlens:
 * HOST int32 [n_seqs + 1] token offsets (cu[0] = 0, cu[n] = T). The offsets
 * reach the GPU through a pinned buffer and its device copy that the call has to
 * itself: it waits for its work on `stream`, so it cannot be captured, and may
 * come from any stream or thread. Up to four such pairs of at most 256 KiB
 * each are kept per device until the process ends. */
hs_status hs_k_attn_prefill(const void* qkv, void* out, const int32_t* cu_seqlens,
                            int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads,
                            int32_t head_dim, void* stream);

/* Attention of one new query per sequence over its paged KV cache (the
 * attention of a decode step: the keys and values cached during prefill and
 * earlier steps are reused). q: bf16 [B][ldq], query head h at column
 * h * head_dim, already rotated; pool: one layer's KV pool, bf16
 * [blocks][K | V][n_kv_heads][16][head_dim] with post-RoPE keys;
 * block_table: device int32 [B][max_blocks] (logical block -> pool block);
 * ctx: device int32 [B], cached tokens of each sequence including the new
 * one (1 <= ctx <= max_ctx); out: bf16 [B][ldo], head h at column
 * h * head_dim. max_ctx (host) sizes the launch. The context is processed in
 * fixed 128-token splits whose partial results go through a workspace that
 * the library allocates per device on first use and grows when needed
 * (calls on one device must not overlap); the call is asynchronous on
 * `stream` and deterministic. */
hs_status hs_k_attn_decode(const void* q, int64_t ldq, const void* pool,
                           const int32_t* block_table, const int32_t* ctx, void* out,
                           int64_t ldo, int32_t B, int32_t n_heads, int32_t n_kv_heads,
                           int32_t head_dim, int32_t max_blocks, int32_t max_ctx,
                           void* stream);

/* The same attention with the decode step's RoPE and cache append folded in
 * (LLM inference: the new token's key and value join the cache and every
 * later step reuses them). qkv: bf16 [B][ldqkv], the QKV projection of each
 * sequence's new token before RoPE (query heads, then key heads, then value
 * heads, head_dim columns each); the new token sits at position ctx - 1 of
 * its sequence and is NOT read from the pool: the call rotates the queries
 * and the new key by the rotate-half RoPE at that position (float32
 * arithmetic, bf16 rounding), attends over the cached tokens plus the new
 * one, and writes the rotated key and the value into the token's slot of
 * pool (block block_table[b][(ctx - 1) / 16], offset (ctx - 1) % 16), which
 * the caller must have allocated. cos_t, sin_t: device float32
 * [max_pos][head_dim / 2], cos and sin of pos * base^(-2 i / head_dim);
 * max_ctx <= max_pos. Other arguments, workspace and errors as for
 * hs_k_attn_decode. */
hs_status hs_k_attn_decode_rope(const void* qkv, int64_t ldqkv, void* pool,
                                const int32_t* block_table, const int32_t* ctx,
                                const float* cos_t, const float* sin_t, int32_t max_pos,
                                void* out, int64_t ldo, int32_t B, int32_t n_heads,
                                int32_t n_kv_heads, int32_t head_dim, int32_t max_blocks,
                                int32_t max_ctx, void* stream);

/* Greedy sampling of the first token and of every decode step (section 2.1:
 * the next token is chosen from the logits of the last position): out[r] =
 * the lowest column index c with logits[r][c] equal to the row's maximum.
 * logits: device float32 [n_rows][n_cols], row-major, 16-byte aligned;
 * out: device int32 [n_rows]. Requires n_rows >= 1 and n_cols >= 1 with
 * n_cols % 4 == 0 (HS_EINVAL otherwise). NaN entries never win; a row of
 * NaN only gives 0x7FFFFFFF. The call allocates a small device buffer for
 * the per-chunk candidates, launches on `stream` (one pass up to 4096 columns,
 * two above), waits for the result and frees the buffer. */
hs_status hs_k_argmax(const float* logits, int32_t n_rows, int32_t n_cols, int32_t* out,
                      void* stream);

/* RMSNorm of `rows` rows of width `hidden`: out = x / sqrt(mean(x^2) + eps) * g,
 * bf16 in and out, float32 arithmetic. */
hs_status hs_k_rmsnorm(const void* x, const void* g, void* out, int32_t rows, int32_t hidden,
                       float eps, void* stream);

/* hs_k_attn_decode without any device allocation, for callers that cannot
 * allocate: code under HIP graph capture, serving loops that must not call
 * hipMalloc, harnesses that forbid it. Arguments, kernels, results (bitwise)
 * and errors are those of hs_k_attn_decode. The split partials live in a
 * static device array of HS_K_ATTN_DECODE_NOALLOC_MAX_FLOATS floats
 * (32 MiB), one per GPU, held until the process ends; a call needing more,
 * B * n_heads * ceil(max_ctx / 128) * (head_dim + 2) floats, returns
 * HS_ERANGE before touching the GPU. Every call on one GPU uses the same
 * array, so calls that overlap in time on one GPU (other streams, other
 * threads) race and give wrong results: order them. */
#define HS_K_ATTN_DECODE_NOALLOC_MAX_FLOATS (8ll * 1024 * 1024)
hs_status hs_k_attn_decode_noalloc(const void* q, int64_t ldq, const void* pool,
                                   const int32_t* block_table, const int32_t* ctx, void* out,
                                   int64_t ldo, int32_t B, int32_t n_heads, int32_t n_kv_heads,
                                   int32_t head_dim, int32_t max_blocks, int32_t max_ctx,
                                   void* stream);

/* ---- Operators of caches beyond one sequence's plain decode step ----
 *
 * Rotation tables for long contexts, rotation and cache append where position
 * and slot differ, decode attention for sequences that share a prefix, decode
 * attention that also accumulates the weight of every cached token, and
 * eviction by that weight. A step of a batch under a cache budget is
 * hs_k_rope_kv, hs_k_attn_decode_weights, then hs_k_kv_evict.
 *
 * Common to them: head_dim is 64 or 128 and n_heads / n_kv_heads 1 to 16. Pools are
 * as in hs_k_attn_decode; pool_blocks is the number of blocks of the pool, and
 * an entry of a block table or a slot outside of it is never followed. bf16
 * matrices and the pool are 16-byte aligned, their row strides multiples of 8
 * elements, int32 and float32 arrays 4-byte aligned. The calls allocate
 * nothing, keep no state and may be captured into a graph; what they need is
 * in `ws`, device memory of the caller, 16-byte aligned, of at least the bytes
 * that the matching _ws function gives (HS_ERANGE below it). ws need not be
 * cleared, and calls that may overlap in time need one each, replays of
 * captured calls too. Outputs overlap neither inputs nor each other but where it
 * says so (HS_EINVAL; they may lie in the gaps of rows whose stride is the same; pools
 * and rotary tables are not looked at). Buffers and the stream belong to the current
 * device. B is at most 65535, prefix_len and max_ctx at most 2^30, pool_blocks 2^27. A
 * call that needs 2^32 threads or more is refused, by its _ws function too: attention has
 * 256 or 512 of them per kv head and split of a sequence (128 tokens or more), rotation one
 * per token and 16 elements of its heads.
 * Results are deterministic. */

/* How the angles of rotary positions are scaled. w_i = base^(-2 i / rot_dim) is
 * the unscaled angle per position of pair i, t_i = original_ctx w_i / 2 pi its
 * turns over the context that the model was trained on. */
enum {
  HS_ROPE_PLAIN = 0,  /* w_i */
  HS_ROPE_LINEAR = 1, /* w_i / factor */
  HS_ROPE_NTK = 2,    /* of base * factor^(rot_dim / (rot_dim - 2)) */
  HS_ROPE_BANDS = 3,  /* s w_i + (1 - s) w_i / factor, s = (t_i - low) / (high - low) cut to [0, 1] */
  HS_ROPE_YARN = 4    /* the same with 1 - s = (i - a) / max(b - a, 0.001) cut to [0, 1],
                       * a = max(0, floor d(high)), b = min(rot_dim - 1, ceil d(low)),
                       * d(x) = rot_dim ln(original_ctx / (2 pi x)) / (2 ln base) */
};
typedef struct {
  int32_t kind;         /* HS_ROPE_* */
  int32_t original_ctx; /* BANDS and YARN: >= 1 */
  double factor;        /* all but PLAIN: > 0, w_i / factor finite */
  double low, high;     /* BANDS and YARN: 0 < low < high */
  double magnitude;     /* cos and sin are multiplied by it (> 0, finite as float32) */
} hs_rope_scaling;

/* cos_t[p][i] = magnitude cos(p w_i'), sin_t[p][i] = magnitude sin(p w_i') for p <
 * max_pos, i < rot_dim / 2: device float32 [max_pos][rot_dim / 2], 16-byte
 * aligned. rot_dim: 8 to 128, a multiple of 8; base > 1; scaling: host, NULL = plain
 * with magnitude 1. The angle per position is formed in float64 and held as a 64-bit
 * fraction of a turn, and entries are within 6 x 2^-24 of their value for it: far
 * positions are as exact as near ones, and small sines as large ones. */
hs_status hs_k_rope_tables(float* cos_t, float* sin_t, int32_t max_pos, int32_t rot_dim,
                           double base, const hs_rope_scaling* scaling, void* stream);

/* Rotation of the first rot_dim elements of every query and key head of T tokens
 * (the rest passes as it is), and append of the rotated keys and the values to
 * the paged cache. qkv: bf16 [T][ldqkv] (query heads, key heads, value heads);
 * pos: device int32 [T]; slot: device int32 [T], block * 16 + offset. A token whose
 * pos is outside [0, max_pos) is an empty row of a padded batch: nothing of it is
 * written. One whose slot is outside the pool is rotated but not appended. Two
 * tokens of a call have different slots. cos_t, sin_t: float32 [max_pos][rot_dim / 2],
 * 16-byte aligned; rot_dim: 16 to head_dim, a multiple of 16. layout 0: pairs
 * (i, i + rot_dim / 2); 1: interleaved, (2 i, 2 i + 1). q_out: bf16 [T][ldq]; k_out:
 * bf16 [T][ldk] rotated keys, or NULL. q_out may be qkv itself, and k_out its key
 * columns, with ldq and ldk equal to ldqkv. Float32 arithmetic, one rounding. */
hs_status hs_k_rope_kv(const void* qkv, int64_t ldqkv, const int32_t* pos, const int32_t* slot,
                       const float* cos_t, const float* sin_t, int32_t max_pos, int32_t rot_dim,
                       int32_t layout, void* q_out, int64_t ldq, void* k_out, int64_t ldk,
                       void* pool, int32_t pool_blocks, int32_t T, int32_t n_heads,
                       int32_t n_kv_heads, int32_t head_dim, void* stream);

/* hs_k_attn_decode for B sequences that share the first prefix_len tokens: the
 * query of each attends over the prefix and then its own ctx[b] cached tokens.
 * prefix: device int32 [ceil(prefix_len / 16)], the prefix's blocks (its last one
 * may be filled in part); block_table, ctx: of each sequence's own tokens, 0 <= ctx
 * <= max_ctx (values outside are cut to it). prefix_len and max_ctx may be 0; with
 * max_ctx 0 block_table may be NULL, with prefix_len 0 prefix may. Tokens of a
 * block outside the pool count as not cached; a sequence without any token gives
 * zeros. hs_k_attn_decode_shared_ws: the workspace. */
hs_status hs_k_attn_decode_shared_ws(int32_t B, int32_t n_heads, int32_t n_kv_heads,
                                     int32_t head_dim, int32_t prefix_len, int32_t max_ctx,
                                     uint64_t* bytes);
hs_status hs_k_attn_decode_shared(const void* q, int64_t ldq, const void* pool,
                                  int32_t pool_blocks, const int32_t* prefix, int32_t prefix_len,
                                  const int32_t* block_table, const int32_t* ctx, void* out,
                                  int64_t ldo, int32_t B, int32_t n_heads, int32_t n_kv_heads,
                                  int32_t head_dim, int32_t max_blocks, int32_t max_ctx, void* ws,
                                  uint64_t ws_bytes, void* stream);

/* The same attention, and the weight that each own token received: with p[h][t]
 * the probability that query head h gave to token t of sequence b,
 *   acc_out[b][k][t] = decay acc[b][k][t] + sum over the query heads h of kv head k of p[h][t]
 * for t < ctx[b] - 1; the newest token, t = ctx[b] - 1, starts at its sum (acc is not
 * read there), and pos[b][k][ctx[b] - 1] = seen[b] - 1, the position of the newest of
 * the seen[b] tokens of the sequence. acc, acc_out: device float32
 * [B][n_kv_heads][acc_stride], acc_stride >= max_ctx; pos: int32 of the same shape, or
 * NULL (seen is then not read); seen: device int32 [B]. acc_out may be acc. What
 * lies at or past ctx[b] is left as it was. decay >= 0, finite. */
hs_status hs_k_attn_decode_weights_ws(int32_t B, int32_t n_heads, int32_t n_kv_heads,
                                      int32_t head_dim, int32_t prefix_len, int32_t max_ctx,
                                      uint64_t* bytes);
hs_status hs_k_attn_decode_weights(const void* q, int64_t ldq, const void* pool,
                                   int32_t pool_blocks, const int32_t* prefix, int32_t prefix_len,
                                   const int32_t* block_table, const int32_t* ctx, void* out,
                                   int64_t ldo, const float* acc, float* acc_out,
                                   int64_t acc_stride, float decay, int32_t* pos,
                                   const int32_t* seen, int32_t B, int32_t n_heads,
                                   int32_t n_kv_heads, int32_t head_dim, int32_t max_blocks,
                                   int32_t max_ctx, void* ws, uint64_t ws_bytes, void* stream);

/* Eviction: of each kv head of each sequence with more than `keep` cached tokens
 * the `keep` best stay: those with pos < sinks or pos >= seen[b] - recent first, then by
 * acc, largest first (a NaN last), then the lower slot (protected ones among
 * themselves by slot alone). The tokens that stay are packed into slots [0, keep):
 * one whose slot is below keep does not move; the j-th slot below keep that became
 * free takes the j-th token that stays at or past keep: its key and value in the
 * pool, its acc and pos. acc, pos: device [B][n_kv_heads][stride]; acc_out, pos_out:
 * [B][n_kv_heads][out_stride], entries t < ctx_out[b] are written (rows of at most keep
 * tokens are copied); they may be acc and pos themselves, with the same stride.
 * ctx_out[b] = min(ctx[b], keep), and may not be ctx. The sequences' own blocks are
 * distinct. stride >= max_ctx, out_stride >= min(keep, max_ctx); keep >= 1, sinks and
 * recent >= 0; min(keep, max_ctx - keep), the moves that a row can have, at most 2^25. A move
 * from or to a block outside the pool is left out. */
hs_status hs_k_kv_evict_ws(int32_t B, int32_t n_kv_heads, int32_t keep, int32_t max_ctx,
                           uint64_t* bytes);
hs_status hs_k_kv_evict(void* pool, int32_t pool_blocks, const int32_t* block_table,
                        const int32_t* ctx, const int32_t* seen, const float* acc,
                        const int32_t* pos, int64_t stride, float* acc_out, int32_t* pos_out,
                        int64_t out_stride, int32_t* ctx_out, int32_t keep, int32_t sinks,
                        int32_t recent, int32_t B, int32_t n_kv_heads, int32_t head_dim,
                        int32_t max_blocks, int32_t max_ctx, void* ws, uint64_t ws_bytes,
                        void* stream);

#ifdef __cplusplus
}
#endif

#endif /* HS_KERNEL_H */
