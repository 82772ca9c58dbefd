/*
 * shotkv.h - C ABI of the MI355X (gfx950) ShotKV KV-cache compression library.
 *
 * ShotKV (arXiv 2502.01941, Section 5 "ShotKV", Eq. 2-9, Algorithm 1) compresses a transformer's KV
 * cache in two phases.  Prefill: every few-shot example ("shot") of the prompt is scored by the
 * attention mass its tokens receive, whole shots are kept in descending score order under a token
 * budget, and the kept K/V rows are compacted into a dense cache that then stays fixed.  Decoding:
 * generated tokens are retained at token level by the attention the current query gives them, and
 * attention runs over the union of the two caches.
 *
 * Conventions for every entry point
 *   - All data pointers are DEVICE pointers owned by the caller.  The library never allocates, frees
 *     or synchronises; it enqueues kernels on `stream` (a hipStream_t passed as void*, NULL = the
 *     default stream) and returns.  Inputs are never written.
 *   - Return value: SHOTKV_OK or a negative SHOTKV_E_* for errors the host can see (null pointer,
 *     unsupported shape, workspace too small, misaligned pointer).  Nothing is enqueued on error.
 *   - Data-dependent errors are reported per problem in a device-side `status` word (SHOTKV_ST_*);
 *     a failed problem keeps nothing (kept_count = 0).
 *   - Tensors are dense, row-major, innermost dimension head_dim; every tensor pointer must be
 *     16-byte aligned.  "dtype" below is cfg->dtype: bf16 (2 bytes) or fp32 (4 bytes).
 *   - Supported shapes: head_dim 64 or 128; n_q_heads = G * n_kv_heads with 1 <= G <= 8, n_q_heads <= 64;
 *     1 <= window <= 64 and G * window <= 256; n_shots <= SHOTKV_MAX_SHOTS; n_tokens <= 2^30 where shots are
 *     scored.
 *   - Two calls that share a workspace or outputs must be ordered on one stream.
 */
#ifndef SHOTKV_H
#define SHOTKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SHOTKV_MAX_SHOTS 4096

#if defined(__GNUC__)
#define SHOTKV_API __attribute__((visibility("default")))
#else
#define SHOTKV_API
#endif

enum { SHOTKV_BF16 = 0, SHOTKV_F32 = 1 };

/* How the ranked walk treats a shot that does not fit (Section 5.1, the paragraph after Eq. 3: shots
 * are taken in descending score order up to the budget).  PREFIX stops at the first misfit (the literal
 * reading, default); FIRST_FIT skips it and continues with lower-ranked shots. */
enum { SHOTKV_SELECT_PREFIX = 0, SHOTKV_SELECT_FIRST_FIT = 1 };

/* Which heads a shot's score sums over.  PER_LAYER is Eq. 3 as printed: all H query heads, one
 * selection per (batch, layer) problem shared by its KV heads.  PER_KV_HEAD restricts the head sum to
 * the G query heads that read a KV head, so every KV head ranks the shots, keeps its own subset under
 * the same budget and owns its own cache ("ragged" caches); in decoding each KV head then also
 * retains its own generated tokens by the attention of its own query group.  In this mode every
 * per-problem output and per-sequence state array gains an H_kv dimension, as noted at each entry
 * point; inputs are unchanged. */
enum { SHOTKV_HEADS_PER_LAYER = 0, SHOTKV_HEADS_PER_KV_HEAD = 1 };

enum {
  SHOTKV_OK = 0,
  SHOTKV_E_NULL = -1,      /* a required pointer is NULL                         */
  SHOTKV_E_SHAPE = -2,     /* unsupported or inconsistent shape / dtype / mode   */
  SHOTKV_E_WORKSPACE = -3, /* workspace_bytes smaller than *_workspace_bytes()   */
  SHOTKV_E_ALIGN = -4,     /* a tensor pointer is not 16-byte aligned            */
  SHOTKV_E_LAUNCH = -5,    /* the HIP runtime refused a launch                   */
  SHOTKV_E_SCRATCH = -6    /* shotkv_decode_step_static: needs more than SHOTKV_STATIC_SCRATCH_BYTES */
};

/* Per-problem device-side status words. */
enum {
  SHOTKV_ST_OK = 0,
  SHOTKV_ST_BAD_OFFSETS = -1,      /* shot offsets not strictly increasing or outside [0, n_tokens] */
  SHOTKV_ST_BUDGET_TOO_SMALL = -2, /* tokens outside every shot already exceed the budget            */
  SHOTKV_ST_NO_FREE_SLOT = -3,     /* decode: the slot pool is full                                  */
  SHOTKV_ST_NO_FREE_PAGE = -4,     /* paged cache: the free stack is too short                       */
  SHOTKV_ST_BAD_LENGTH = -5,       /* paged cache: a length that is negative or does not fit         */
  SHOTKV_ST_BAD_TREE = -6          /* drafted trees: a parent that is not before its token           */
};

typedef struct {
  int32_t n_q_heads;   /* H                                                       */
  int32_t n_kv_heads;  /* H_kv; query head h reads KV head h / (H / H_kv)         */
  int32_t head_dim;    /* D                                                       */
  int32_t window;      /* W: observation-window queries = last W prefill positions */
  int32_t dtype;       /* SHOTKV_BF16 or SHOTKV_F32: element type of Q, K, V      */
  float   sm_scale;    /* logits = sm_scale * <q, k>                              */
  int32_t select_mode; /* SHOTKV_SELECT_*                                          */
  int32_t head_mode;   /* SHOTKV_HEADS_*                                           */
  /* Optional per-kernel timing for benchmarks (not part of the method): NULL, or a host array of
   * 2 * SHOTKV_KERNEL_KINDS hipEvent_t handles created and owned by the caller.  A call records
   * events [2 * kind] and [2 * kind + 1] on its stream around each kernel of that kind it enqueues;
   * the caller synchronises and reads elapsed times.  The library creates no objects and keeps no
   * state between calls.  Kinds, in order: chunk plan, score, row statistics, chunk mass, shot scores
   * and selection, compaction, decode partial, decode finish, V packing, fused attention.  Chunk plan and row
   * statistics have no kernels of their own (scoring and fused attention find their chunks themselves, chunk mass
   * the row statistics): their events are recorded with nothing in between, so the kinds add up to the call.  So are
   * compaction's where few rows are copied (up to 48 MB read and written in a call): the kernel that selects makes the
   * copies as well, and its kind has the time of both. */
  void* const* timing_events;
} shotkv_config;

SHOTKV_API const char* shotkv_strerror(int code);
SHOTKV_API int32_t shotkv_abi_version(void);

#define SHOTKV_KERNEL_KINDS 10

/* Bytes of device workspace shotkv_prefill_compress / _scores / _select_and_compact need for P
 * problems of n_tokens tokens and n_shots shots.  0 if the shape is unsupported. */
SHOTKV_API size_t shotkv_prefill_workspace_bytes(const shotkv_config* cfg, int32_t P, int32_t n_tokens,
                                      int32_t n_shots);

/*
 * Prefill compression (Section 5.1, Eq. 3-6; Algorithm 1, phase 1) of P independent (batch, layer)
 * problems that share one shape.
 *
 * Per problem: (1) softmax attention of the W window queries of every query head over the n_tokens
 * keys of its KV head, causal inside the window (query j sits at position n_tokens-W+j); (2) the
 * weights are summed over all H heads and W queries per key and averaged over each shot's tokens,
 * Score(s_i) of Eq. 3; (3) shots are ranked by score descending, ties to the lower index, and whole
 * shots are kept while they fit (Eq. 5-6); tokens outside every shot - before shot_offsets[0] and
 * from shot_offsets[n_shots] on - are always kept and are charged to the budget first; (4) the kept
 * rows of K and V are copied, in ascending position, into the dense output (Eq. 4).
 *
 *   q_obs          [P][H][W][D] dtype          window queries, unscaled
 *   k, v           [P][H_kv][n_tokens][D] dtype
 *   shot_offsets   [P][n_shots+1] int32        shot i = [off[i], off[i+1]); strictly increasing
 *   budget_tokens  [P] int32                   N_budget: most tokens a problem may retain
 *   k_out, v_out   [P][H_kv][cap][D] dtype     rows [0, kept_count) written, the rest untouched
 *   cap            rows per head in k_out/v_out; must be >= every budget (larger budgets are clamped)
 *   kept_positions [P][cap] int32              original position of each output row, ascending
 *   kept_count     [P] int32
 *   shot_scores    [P][n_shots] float          Score(s_i)                       (may be NULL)
 *   shot_selected  [P][n_shots] uint8          1 = kept                          (may be NULL)
 *   status         [P] int32                   SHOTKV_ST_*
 *
 * With cfg->head_mode = SHOTKV_HEADS_PER_KV_HEAD steps (2)-(4) run once per KV head over that head's
 * G query heads, and kept_positions is [P][H_kv][cap], kept_count [P][H_kv], shot_scores
 * [P][H_kv][n_shots], shot_selected [P][H_kv][n_shots], status [P][H_kv]; head g of k_out/v_out holds
 * kept_count[p][g] rows.
 */
SHOTKV_API int shotkv_prefill_compress(const shotkv_config* cfg, int32_t P, int32_t n_tokens, int32_t n_shots,
                            const void* q_obs, const void* k, const void* v,
                            const int32_t* shot_offsets, const int32_t* budget_tokens,
                            void* k_out, void* v_out, int32_t cap,
                            int32_t* kept_positions, int32_t* kept_count,
                            float* shot_scores, uint8_t* shot_selected, int32_t* status,
                            void* workspace, size_t workspace_bytes, void* stream);

/* The scoring half alone (steps 1-2 above; Eq. 3): writes shot_scores [P][n_shots] and status
 * ([P][H_kv][n_shots] and [P][H_kv] in per-KV-head mode). */
SHOTKV_API int shotkv_prefill_scores(const shotkv_config* cfg, int32_t P, int32_t n_tokens, int32_t n_shots,
                          const void* q_obs, const void* k, const int32_t* shot_offsets,
                          float* shot_scores, int32_t* status,
                          void* workspace, size_t workspace_bytes, void* stream);

/* The selection and compaction half alone (steps 3-4 above; Eq. 4-6) from caller-supplied scores.
 * Arguments as in shotkv_prefill_compress; shot_scores is an input here.  -0 ranks with +0; a NaN has no
 * rank and is placed by its bit pattern (deterministic, otherwise unspecified). */
SHOTKV_API int shotkv_select_and_compact(const shotkv_config* cfg, int32_t P, int32_t n_tokens, int32_t n_shots,
                              const float* shot_scores, const void* k, const void* v,
                              const int32_t* shot_offsets, const int32_t* budget_tokens,
                              void* k_out, void* v_out, int32_t cap,
                              int32_t* kept_positions, int32_t* kept_count,
                              uint8_t* shot_selected, int32_t* status,
                              void* workspace, size_t workspace_bytes, void* stream);

/*
 * Prefill compression fused into the prompt's own attention pass (Section 5.1, Eq. 3-6; the appendix on
 * limitations names kernel-level optimisation of the scoring step as open).  The prefill phase of a
 * decoder computes causal attention for every prompt position anyway, and the last W query rows of that
 * pass are the observation-window rows whose weights Eq. 3 pools.  This entry point computes
 *
 *   attn_out [P][H][n_tokens][D] float   softmax(sm_scale * Q K^T) V, causal, query head h on KV head h / G
 *
 * for the whole prompt and takes the window rows' weights from the same pass, so K is not read a second
 * time for scoring; steps (2)-(4) of shotkv_prefill_compress then run unchanged.
 *
 *   q   [P][H][n_tokens][D] dtype   all query rows of the layer (the last W are the window queries)
 *
 * Every other argument is as in shotkv_prefill_compress, and so is every result: shot_scores agree with
 * that entry point's to rounding (both head modes).  Shapes: bf16, head_dim 128; anything else returns
 * SHOTKV_E_SHAPE.  The workspace (shotkv_prefill_attention_workspace_bytes) also holds a packed copy of V.
 * Accuracy of attn_out: Q K^T in bf16 with fp32 accumulation, the weighted sum of V rows in fp16 (weights
 * with 11 significant bits, V scaled per KV-head plane by an exact power of two so that any finite bf16
 * values are representable) with fp32 accumulation and fp32 weight sums: each output row is within 1e-3 of
 * its largest magnitude of the exact result.
 */
SHOTKV_API size_t shotkv_prefill_attention_workspace_bytes(const shotkv_config* cfg, int32_t P, int32_t n_tokens,
                                                int32_t n_shots);
SHOTKV_API int shotkv_prefill_attention_compress(const shotkv_config* cfg, int32_t P, int32_t n_tokens, int32_t n_shots,
                                      const void* q, const void* k, const void* v,
                                      const int32_t* shot_offsets, const int32_t* budget_tokens,
                                      float* attn_out, void* k_out, void* v_out, int32_t cap,
                                      int32_t* kept_positions, int32_t* kept_count, float* shot_scores,
                                      uint8_t* shot_selected, int32_t* status, void* workspace,
                                      size_t workspace_bytes, void* stream);

/*
 * Decode state of one layer for S sequences: caller-owned device buffers.
 * The prefill cache is what shotkv_prefill_compress produced and is never written here (Section 5.1,
 * Eq. 2: the prefill part is compressed one time only and kept as it is while decoding).  Generated
 * tokens live in a pool of n_slots slots per
 * sequence; slot_pos holds the generated-token index in each slot, -1 when free (initialise to -1).
 * n_slots must be >= decode_budget + 1 unless the caller guarantees fewer steps than n_slots.
 * Rows of the prefill cache past prefill_count may hold anything: they may be fetched but never
 * influence a result.  decode_budget may stay or grow from step to step, e.g. ceil(r_d * (step_index +
 * 1)) for the ratio form of Eq. 8; a step evicts at most one token, so a budget that shrinks is not
 * honoured (the cache keeps the size it has).
 * In per-KV-head mode prefill_count is [S][H_kv] and slot_pos [S][H_kv][n_slots]: every KV head has
 * its own live row count and its own slot map.
 */
typedef struct {
  const void*    k_prefill;      /* [S][H_kv][cap][D] dtype                                   */
  const void*    v_prefill;      /* [S][H_kv][cap][D] dtype                                   */
  const int32_t* prefill_count;  /* [S] live rows in the prefill cache, <= cap                */
  void*          k_dec;          /* [S][H_kv][n_slots][D] dtype                               */
  void*          v_dec;          /* [S][H_kv][n_slots][D] dtype                               */
  int32_t*       slot_pos;       /* [S][n_slots]                                              */
  int32_t        cap;
  int32_t        n_slots;
  int32_t        decode_budget;  /* B_d; INT32_MAX = never evict (prefill-only ablation)      */
} shotkv_decode_state;

SHOTKV_API size_t shotkv_decode_workspace_bytes(const shotkv_config* cfg, int32_t S, int32_t cap, int32_t n_slots);

/*
 * One decoding step (Section 5.1, Eq. 7-9; Algorithm 1, phase 2) for S sequences.
 *
 * Per sequence: the new token's k_new/v_new go into the lowest-numbered free slot (slot_pos becomes
 * step_index); every query head attends over the live prefill rows plus the occupied slots (Eq. 9);
 * Score(t) = sum over heads of the weight given to decode token t at this step (Eq. 7); if the
 * decode cache now holds more than decode_budget tokens, the lowest-scored earlier token is evicted
 * (the token just appended is exempt; among equal scores the newest goes) and its slot freed (Eq. 8
 * with a fixed capacity).
 *
 *   q_new        [S][H][D] dtype       k_new, v_new [S][H_kv][D] dtype
 *   out          [S][H][D] float       attention output                          (required)
 *   token_scores [S][n_slots] float    Score(t) per slot, 0 on free slots         (may be NULL)
 *   evicted_pos  [S] int32             token index evicted this step, else -1     (may be NULL)
 *   status       [S] int32             SHOTKV_ST_*                                (required)
 *
 * In per-KV-head mode Eq. 7 sums over the G query heads of a KV head, Eq. 8 runs per KV head, and
 * token_scores is [S][H_kv][n_slots], evicted_pos and status [S][H_kv].
 */
SHOTKV_API int shotkv_decode_step(const shotkv_config* cfg, int32_t S, const shotkv_decode_state* st,
                       int32_t step_index, const void* q_new, const void* k_new, const void* v_new,
                       float* out, float* token_scores, int32_t* evicted_pos, int32_t* status,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * shotkv_decode_step without a workspace argument, for callers that cannot allocate device memory:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same kernels,
 * same arguments, same results as shotkv_decode_step; the workspace is a buffer of
 * SHOTKV_STATIC_SCRATCH_BYTES that is part of the library's device image (one copy per GPU, held until
 * the process ends).  The call allocates and frees nothing and creates no objects.  The first call on
 * a GPU looks up the buffer's address (make that call outside a graph capture).
 *
 * Limit: returns SHOTKV_E_SCRATCH, and enqueues nothing, when shotkv_decode_workspace_bytes(cfg, S,
 * st->cap, st->n_slots) exceeds SHOTKV_STATIC_SCRATCH_BYTES (8 MiB holds e.g. 16 sequences with 32
 * query heads, head_dim 128, a 4096-row prefill cache and 1025 slots).
 * All calls on one GPU share the buffer, whatever their stream: calls that may overlap in time race
 * with each other; order them on one stream or with events.  The buffer keeps the last call's
 * contents; a step reads nothing from it that it has not written itself.
 */
#define SHOTKV_STATIC_SCRATCH_BYTES (8u << 20)
SHOTKV_API int shotkv_decode_step_static(const shotkv_config* cfg, int32_t S, const shotkv_decode_state* st,
                              int32_t step_index, const void* q_new, const void* k_new, const void* v_new,
                              float* out, float* token_scores, int32_t* evicted_pos, int32_t* status,
                              void* stream);

/*
 * The paged 4-bit cache.
 *
 * Compressed prompts and the tokens generated after them, of many requests, in one pool of pages.  A page holds
 * `page_size` tokens (32, 64, 128, ... 32768) of all KV heads; a request's pages are listed in its row of the block table.
 * A slot is page * page_size + offset, the place of one token.  Rows of keys and values are held in groups of 32
 * channels: 4-bit codes (a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6) that share a power of two.
 *
 *   scale  of a group whose largest magnitude is a: 2^e with the least e for which a <= 7 * 2^e, -126 <= e <= 125,
 *          stored as the byte e + 127.  A value is then off by at most half of the widest step (2^e; magnitudes of
 *          2^127 or more, which nothing above 6 * 2^125 can stand for, by more).  A group with a value that is not
 *          finite has the byte 255 and reads back as NaN.
 *   code   the magnitude nearest to |x| * 2^-e, ties to the even code, and the sign in bit 3.
 *   page   [n_kv_heads][page_size / 32] blocks of 32 tokens.  A block has 34 * D bytes: key codes [32 tokens][D / 2],
 *          value codes [8 quads of tokens][D / 8][4 tokens][4], key scales [32 tokens][D / 32], value scales
 *          [8 quads][D / 32][4 tokens].  Channel 2 i is the low half of byte i of its row.
 *
 * Head layouts and types are those of the configuration (head_dim 64 or 128, n_q_heads = G * n_kv_heads with G <= 8,
 * n_q_heads <= 64); window, select_mode and head_mode are not looked at.  Caches that differ from KV head to KV head
 * (SHOTKV_HEADS_PER_KV_HEAD) are requests of their own with one KV head each.  None of these entry points records
 * timing events.  What a table or a map says is checked on the device: slots, pages and positions outside of their
 * range are taken for none, never read or written.  Up to 65535 requests, 2^28 tokens in a batch (of none, nothing is
 * done), 2^30 tokens in a row of a block table (max_pages * page_size) and 2^29 rows of queries in a request (the lesser of
 * max_q_len and T, times n_q_heads).
 */
typedef struct {
  void*   pages;      /* [n_pages][shotkv_kv4_page_bytes] device, 16-byte aligned */
  int32_t n_pages;
  int32_t page_size;  /* tokens of a page: a power of two from 32 to 32768; n_pages * page_size <= 2^31 - 1 */
} shotkv_kv4_cache;

/* Rows of head_dim elements of cfg->dtype for T tokens of some heads, anywhere: element (t, h, d) is
 * data[(t / seq_tokens) * seq_stride + (t % seq_tokens) * token_stride + h * head_stride + d], strides in elements.
 * Every row starts at a multiple of 16 bytes.  [T][heads][D] has seq_tokens = T and strides (any, heads * D, D);
 * a cache of shotkv_prefill_compress, [P][H_kv][cap][D], seq_tokens = cap and strides (H_kv * cap * D, D, cap * D). */
typedef struct {
  void*   data;
  int64_t seq_stride, token_stride, head_stride;
  int32_t seq_tokens;
} shotkv_rows;

/* Bytes of a page, n_kv_heads * page_size * 17 / 16 * head_dim; 0 if the shape is unsupported. */
SHOTKV_API size_t shotkv_kv4_page_bytes(int32_t page_size, int32_t n_kv_heads, int32_t head_dim);

/*
 * Pages for the new tokens of R requests, and where each token goes.
 *
 * Request r holds cached_lens[r] tokens in the first ceil(cached_lens[r] / page_size) pages of its row and is to take
 * new_lens[r] more.  Pages come off the top of the free stack in the order of the requests: with n[r] pages needed
 * and s[r] = n[0] + ... + n[r - 1], page j of request r is free_pages[free_count - 1 - s[r] - j].
 *
 *   cached_lens, new_lens  [R] int32
 *   pos_start     [R] int32 or NULL      position of each request's first new token; NULL: cached_lens (a compressed
 *                                        prompt has fewer tokens in the cache than positions behind it)
 *   free_pages    [stack_size] int32     the free stack, not written
 *   free_count    [1] int32              pages on it; stack_size counts if it is more
 *   block_table   [R][max_pages] int32   entries of new pages are written, the others stay
 *   free_left     [1] int32              pages left on the stack; not the same word as free_count
 *   seq_lens      [R] int32              tokens with the new ones; not the same array as cached_lens
 *   query_start   [R + 1] int32          first new token of each request in a batch without gaps, and their number
 *   slot_map, token_pos  [T] int32       slot and position of every token of the batch, -1 where there is none
 *   request_tokens  0: token i of request r is number query_start[r] + i of the batch.  Otherwise a batch of equal
 *                   shares, in which it is number r * request_tokens + i, for rows that are stored as they are
 *                   (shotkv_prefill_compress's).  query_start is as it is without, and not that batch's:
 *                   shotkv_kv4_attention takes batches without gaps only
 *   status        [R] int32              SHOTKV_ST_OK; SHOTKV_ST_NO_FREE_PAGE: pages are needed and the stack ends
 *                 before them; SHOTKV_ST_BAD_LENGTH: a negative length, more pages than max_pages, or more tokens
 *                 than the batch (its share) holds.  Requests with either keep their length, and their new
 *                 tokens have no slot (their rows of the batch stay theirs, a negative new_lens apart).  The status is
 *                 the only sign of that: shotkv_qk_norm_rope makes zeros of such rows, and shotkv_kv4_attention takes
 *                 them for the last tokens of what the request held before; its output there means nothing.
 */
SHOTKV_API int shotkv_pages_plan(int32_t R, int32_t page_size, int32_t max_pages, const int32_t* cached_lens,
                                 const int32_t* new_lens, const int32_t* pos_start, const int32_t* free_pages,
                                 int32_t stack_size, const int32_t* free_count, int32_t* block_table,
                                 int32_t* free_left, int32_t* seq_lens, int32_t* query_start, int32_t T,
                                 int32_t request_tokens, int32_t* slot_map, int32_t* token_pos, int32_t* status,
                                 void* stream);

/* Gives the pages of finished requests back: request r with finished[r] != 0 has its seq_lens[r] set to 0 and its row
 * of the block table to -1, and its ceil(seq_lens[r] / page_size) pages go onto the stack, so that a release of all
 * that a plan gave, to requests that held nothing before, leaves the stack as it was: page j of request r to
 * free_pages[free_count + total - 1 - s[r] - j], s[r] the pages of the finished requests before r.  free_pages has
 * room for stack_size pages; pages that would pass it are dropped (a table that is sound never comes to that).
 * finished [R] uint8; free_count [1] is updated.
 * Entries below 0 are no pages and are left out, and not counted.  All others go onto the stack as often as they
 * are listed, whoever else lists them: where requests share pages, the caller puts -1 in the place of those that stay in
 * use before it releases a request, or they would be handed out twice. */
SHOTKV_API int shotkv_pages_release(int32_t R, int32_t page_size, int32_t max_pages, const uint8_t* finished,
                                    int32_t* seq_lens, int32_t* block_table, int32_t* free_pages, int32_t stack_size,
                                    int32_t* free_count, void* stream);

/* Rotation and norms of shotkv_qk_norm_rope: caller-owned device arrays. */
typedef struct {
  const float*   table;        /* [n_positions][rot_dim]: cosines of the rot_dim / 2 angles, then their sines */
  int32_t        n_positions;
  int32_t        rot_dim;      /* channels that turn: a multiple of 16, at most head_dim; the rest stay */
  int32_t        interleaved;  /* pair i is channels (2 i, 2 i + 1) if set, (i, i + rot_dim / 2) if not */
  float          eps;
  const void*    q_weight;     /* [D] dtype, or NULL: queries are not normalised */
  const void*    k_weight;     /* [D] dtype, or NULL: keys are not normalised */
} shotkv_rope;

/*
 * Norms and rotation of the queries and keys of T tokens, and the new tokens' place in the cache, in one pass.
 * Per token and head: x <- x / sqrt(mean(x^2) + eps) * weight, then each pair (a, b) <- (a cos - b sin, b cos + a sin)
 * with the angles of the token's position; in 32 bits, rounded once to cfg->dtype.
 *
 *   token_pos     [T] int32   a token whose position is outside [0, n_positions) is padding: its output rows are
 *                             zeros and it is not stored
 *   q, q_out      n_q_heads rows per token
 *   k             n_kv_heads rows per token
 *   k_out         as k, or NULL (the keys then only go into the cache)
 *   v, cache, slot_map  [T] int32 slots: the keys (as rounded to cfg->dtype) and values are stored as
 *                             shotkv_kv4_store does; all three or none.  One of k_out and cache is needed.
 */
SHOTKV_API int shotkv_qk_norm_rope(const shotkv_config* cfg, int32_t T, const shotkv_rope* rope,
                                   const int32_t* token_pos, const shotkv_rows* q, const shotkv_rows* k,
                                   const shotkv_rows* q_out, const shotkv_rows* k_out, const shotkv_rows* v,
                                   const shotkv_kv4_cache* cache, const int32_t* slot_map, void* stream);

/* Keys and values of T tokens into the cache, n_kv_heads rows per token each; tokens without a slot are left out.
 * Of two tokens with one slot either may win, in parts. */
SHOTKV_API int shotkv_kv4_store(const shotkv_config* cfg, int32_t T, const shotkv_rows* k, const shotkv_rows* v,
                                const shotkv_kv4_cache* cache, const int32_t* slot_map, void* stream);

/* Keys and values of T tokens out of the cache, as rows of cfg->dtype; zeros for tokens without a slot. */
SHOTKV_API int shotkv_kv4_load(const shotkv_config* cfg, int32_t T, const shotkv_kv4_cache* cache,
                               const int32_t* slot_map, const shotkv_rows* k, const shotkv_rows* v, void* stream);

/*
 * Attention of R requests' new tokens over their cached tokens (their own among them): out = softmax(sm_scale q K^T) V
 * with keys and values as the cache holds them.  With n new tokens in a request of len tokens, query i sees the keys
 * [0, len - n + i].  A query that sees none has an output of zeros and an lse of -infinity; one whose logits are all -infinity, or
 * one of which is infinity or NaN, is NaN in both; one that sees a value that is not finite is NaN in the 32 channels of its
 * group, whatever the value's weight.
 *
 *   max_q_len    most new tokens of a request (of more the first max_q_len are taken, and see what they see among all;
 *                the rows of those that follow are left unwritten)
 *   block_table  [R][max_pages] int32;  lengths past max_pages * page_size are cut
 *   seq_lens     [R] int32;  query_start [R + 1] int32, ascending (entries outside [0, T] count as 0 or T), or NULL: one
 *                token per request (T = R)
 *   q, out       n_q_heads rows per token, cfg->dtype.  lse [T][n_q_heads] float or NULL: natural logarithm of the
 *                sum of exp(sm_scale q.k) over the keys that the query sees.  Rows of tokens that no request has (before
 *                query_start[0], from query_start[R] on) are left unwritten in both
 *
 * Products are of bf16 factors that hold keys and values exactly, summed in 32 bits; weights are taken as the sum of two
 * bf16 numbers (2^-16 off at most), and fp32 queries and the weights of fp32 outputs as the sum of three.
 */
SHOTKV_API size_t shotkv_kv4_attention_workspace_bytes(const shotkv_config* cfg, int32_t R, int32_t T, int32_t max_q_len,
                                                       int32_t page_size, int32_t max_pages);
SHOTKV_API int shotkv_kv4_attention(const shotkv_config* cfg, int32_t R, int32_t T, int32_t max_q_len,
                                    const shotkv_kv4_cache* cache, const int32_t* block_table, int32_t max_pages,
                                    const int32_t* seq_lens, const int32_t* query_start, const shotkv_rows* q,
                                    const shotkv_rows* out, float* lse, void* workspace, size_t workspace_bytes,
                                    void* stream);

/*
 * The same attention with a sliding window and a few first tokens that stay visible.  With n new tokens in a request of len
 * tokens, query i is at position p = len - n + i and sees the keys j <= p that have j > p - window or j < n_sinks.  Positions
 * count the tokens of the cache.
 *
 *   window    keys up to and with its own that a query sees: 1 or more (2^30 and more are all)
 *   n_sinks   first tokens of the request that every query sees as well: 0 or more
 *
 * Blocks of 32 tokens of which no new token sees a key are not read, so their pages need not be there (shotkv_pages_trim);
 * what else is in such a page, or behind the window in one that is read, reaches no result, whatever it is.  (Scale bytes of 253
 * and 254 are written by no store.  With codes that take them past the largest number of bf16 they are infinite or NaN to the queries that
 * see them.)  All other arguments, limits and results are those of shotkv_kv4_attention, and so are the products.
 */
SHOTKV_API size_t shotkv_kv4_window_attention_workspace_bytes(const shotkv_config* cfg, int32_t R, int32_t T, int32_t max_q_len,
                                                              int32_t page_size, int32_t max_pages, int32_t window, int32_t n_sinks);
SHOTKV_API int shotkv_kv4_window_attention(const shotkv_config* cfg, int32_t R, int32_t T, int32_t max_q_len,
                                           const shotkv_kv4_cache* cache, const int32_t* block_table, int32_t max_pages,
                                           const int32_t* seq_lens, const int32_t* query_start, int32_t window, int32_t n_sinks,
                                           const shotkv_rows* q, const shotkv_rows* out, float* lse, void* workspace,
                                           size_t workspace_bytes, void* stream);

/*
 * The same attention for drafted tokens that form a tree (or any other order among themselves).  The n new tokens of a request
 * of len tokens are the last n of its cache.  Query i sees the len - n tokens before them and those of the new tokens whose
 * bits are set in its row of tree_mask: bit j % 32 of word j / 32 is token j of the same request, itself among them only
 * if its own is set.  Bits of tokens that the request does not have count for nothing, and tokens from 32 * mask_words on are
 * seen by none.  What a query does not see does not reach it, whatever it is.
 *
 *   tree_mask [T][mask_words] uint32 (shotkv_tree_plan makes them);  mask_words  1 to 32
 *   window    0: no window.  Otherwise query i is at position p = len - n + (bits that count in its row) - 1, and sees those
 *             of the tokens before the drafts that have j > p - window or j < n_sinks.  The drafts' bits are taken as they are
 *   max_q_len as above, and the first max_q_len tokens of a request still see what their bits say among all
 *
 * All other arguments, limits and results are those of shotkv_kv4_attention; one token per request (query_start NULL) is a
 * tree of one, whose bit says whether it sees itself.
 */
SHOTKV_API size_t shotkv_kv4_tree_attention_workspace_bytes(const shotkv_config* cfg, int32_t R, int32_t T, int32_t max_q_len,
                                                            int32_t page_size, int32_t max_pages, int32_t window, int32_t n_sinks);
SHOTKV_API int shotkv_kv4_tree_attention(const shotkv_config* cfg, int32_t R, int32_t T, int32_t max_q_len,
                                         const shotkv_kv4_cache* cache, const int32_t* block_table, int32_t max_pages,
                                         const int32_t* seq_lens, const int32_t* query_start, const uint32_t* tree_mask,
                                         int32_t mask_words, int32_t window, int32_t n_sinks, const shotkv_rows* q,
                                         const shotkv_rows* out, float* lse, void* workspace, size_t workspace_bytes,
                                         void* stream);

/*
 * What drafted tokens see, and their positions, from their parents.
 *
 *   query_start [R + 1] int32   first token of each request in the batch, as shotkv_pages_plan leaves it (entries outside
 *                               [0, T] count as 0 or T)
 *   parents     [T] int32       number of a token's parent in its request, less than its own; below 0: it follows what is cached
 *   pos_start   [R] int32       position of the tokens without a parent
 *   tree_mask   [T][mask_words] uint32   bits of a token's ancestors and of itself;  mask_words  1 to 32
 *   token_pos   [T] int32       pos_start and one more for each ancestor (past 2^31 - 1: -1, padding to shotkv_qk_norm_rope);
 *                               may be a plan's, whose positions count the drafts as if they came one after the other
 *   status      [R] int32       SHOTKV_ST_OK; SHOTKV_ST_BAD_TREE: a parent that is not before its token; SHOTKV_ST_BAD_LENGTH: more than
 *                               32 * mask_words tokens.  Rows of requests with either, and of no request (before
 *                               query_start[0], from query_start[R] on), have no bits and the position -1
 */
SHOTKV_API int shotkv_tree_plan(int32_t R, int32_t T, const int32_t* query_start, const int32_t* parents, const int32_t* pos_start,
                                int32_t mask_words, uint32_t* tree_mask, int32_t* token_pos, int32_t* status, void* stream);

/*
 * The drafted tokens that the model's own choices confirm, and their rows to the front of the drafts.
 *
 * Token 0 of a request is the one chosen in the step before; it is always kept.  From a token that is kept the one after it is
 * its child (the one of the lowest number, where several are) whose id the model chose there; the first token without such
 * a child is the last, and what the model chose after it is the request's next token 0.  The row of the j-th token kept goes
 * to the place of token j, so that the request's cache is without gaps; the rows behind them are left as they are or hold
 * what they held before others moved.
 *
 *   query_start, parents   as above (of the first token the parent does not matter; one that is not before its token is nobody's)
 *   tokens      [T] int32           ids of the drafted tokens
 *   chosen      [T] int32           ids that the model chose after each; below 0: none
 *   cached_lens [R] int32           tokens of each request without the drafts
 *   path        [R][max_path] int32 numbers of the tokens kept, ascending, then -1.  No more than max_path (1 to 2^28) are kept
 *   accepted    [R] int32           how many
 *   next_token  [R] int32           what the model chose after the last of them; -1: none is kept
 *   kept_lens   [R] int32           cached_lens + accepted; may be cached_lens itself
 *   cache, n_kv_heads, head_dim, layers   the pool whose rows move: n_pages / layers pages of each layer behind those of the
 *                                   layer before, with one block table and slot map for all of them.  NULL: no rows move
 *   slot_map    [T] int32           slots of the drafts in the first layer (shotkv_pages_plan's).  Rows from and to slots outside
 *                                   of it are not moved, and a request whose token 0 has none keeps no token
 *
 * Layers in pools of their own take a call each; as kept_lens then take an array other than cached_lens.
 *
 * Drafts are followed by their parents and slots alone.  Those of a request that shotkv_tree_plan refuses have the position -1, so
 * shotkv_qk_norm_rope does not store them, and no bits, while shotkv_pages_plan has given them slots: they must not be kept.
 * shotkv_tree_keep_planned sees to that.
 */
SHOTKV_API int shotkv_tree_keep(int32_t R, int32_t T, const int32_t* query_start, const int32_t* parents, const int32_t* tokens,
                                const int32_t* chosen, const int32_t* cached_lens, int32_t max_path, int32_t* path,
                                int32_t* accepted, int32_t* next_token, int32_t* kept_lens, const shotkv_kv4_cache* cache,
                                int32_t n_kv_heads, int32_t head_dim, int32_t layers, const int32_t* slot_map, void* stream);

/* The same for drafts of a plan: of requests whose status [R] int32 (shotkv_tree_plan's) is not SHOTKV_ST_OK no token is kept (a path
 * of -1, none accepted, next_token -1, kept_lens the cached_lens) and no row is moved.  It is none of the arrays that are written. */
SHOTKV_API int shotkv_tree_keep_planned(int32_t R, int32_t T, const int32_t* query_start, const int32_t* parents, const int32_t* tokens,
                                        const int32_t* chosen, const int32_t* cached_lens, int32_t max_path, int32_t* path,
                                        int32_t* accepted, int32_t* next_token, int32_t* kept_lens, const shotkv_kv4_cache* cache,
                                        int32_t n_kv_heads, int32_t head_dim, int32_t layers, const int32_t* slot_map,
                                        const int32_t* status, void* stream);

/*
 * Gives the pages back of which no token will be seen again: of the first ceil(held_lens[r] / page_size) entries of a
 * request's row those behind its seq_lens[r] tokens, and those whose tokens are all n_sinks or more and all outside of the
 * window of the token that comes next (at position seq_lens[r]).  Entries that go back become -1; entries below 0 are no pages.
 * Pages go onto the stack so that the first of the first request is on top: number i of them to
 * free_pages[free_count + their number - 1 - i]; pages that would pass stack_size are dropped.
 *
 *   held_lens, seq_lens  [R] int32   tokens that the row has pages for, and those that stay (below 0 count as 0, past
 *                                    max_pages * page_size as that)
 *   window, n_sinks      window 0: none, only what is behind the end goes back
 *   free_left  [1] int32             pages on the stack then; not the same word as free_count, which is not written
 *   given_back [R] int32             pages of each request that went back.  It and free_left are none of the other arrays
 *
 * With a window it is for tables over which every call of attention has this window or a shorter one, and these sinks or fewer:
 * others would take the tokens of the pages that went back for none, without a sign of it.  Layers that see all tokens have a table
 * of their own.  Pages that several requests list go back as often as they are given back: put -1 in the place of those that stay in use.
 */
SHOTKV_API int shotkv_pages_trim(int32_t R, int32_t page_size, int32_t max_pages, const int32_t* held_lens, const int32_t* seq_lens,
                                 int32_t window, int32_t n_sinks, int32_t* block_table, int32_t* free_pages, int32_t stack_size,
                                 const int32_t* free_count, int32_t* free_left, int32_t* given_back, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SHOTKV_H */
