// C ABI of the paged 4-bit cache: argument checks and launches.  Every entry point only enqueues work on the caller's
// stream; nothing is allocated and nothing is kept between calls.
#include "kv4_attention.hpp"

namespace shotkv {

namespace {

constexpr int kMaxRequests = 65535;
constexpr int kMaxTokens = 1 << 28;  // of a batch: rows times heads stay clear of 32-bit overflow
constexpr int kMaxLength = 1 << 30;  // of a request: positions of keys, and blocks past the last one, too
// (token, query head) rows of a request: tiles of 128 of them, times the 2^25 blocks of 32 tokens of the longest cache, stay below
// the 2^48 that sums over a wave's requests take each.
constexpr long long kMaxRows = 1ll << 29;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int log2_page(int page_size) {
  for (int s = 5; s <= 15; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

int check_heads(const shotkv_config* cfg) {
  if (!cfg) return SHOTKV_E_NULL;
  if (cfg->dtype != SHOTKV_BF16 && cfg->dtype != SHOTKV_F32) return SHOTKV_E_SHAPE;
  if (cfg->head_dim != 64 && cfg->head_dim != 128) return SHOTKV_E_SHAPE;
  if (cfg->n_kv_heads < 1 || cfg->n_q_heads < 1 || cfg->n_q_heads > 64 || cfg->n_q_heads % cfg->n_kv_heads) return SHOTKV_E_SHAPE;
  return cfg->n_q_heads / cfg->n_kv_heads > 8 ? SHOTKV_E_SHAPE : SHOTKV_OK;
}

int check_cache(const shotkv_config* cfg, const shotkv_kv4_cache* cache, Kv4Pages* out) {
  if (!cache) return SHOTKV_E_NULL;
  const int shift = log2_page(cache->page_size);
  if (shift < 0 || cache->n_pages < 1 || static_cast<long long>(cache->n_pages) << shift > 0x7fffffffLL) return SHOTKV_E_SHAPE;
  if (!cache->pages) return SHOTKV_E_NULL;
  if (!aligned16(cache->pages)) return SHOTKV_E_ALIGN;
  out->base = static_cast<char*>(cache->pages);
  out->n_pages = cache->n_pages;
  out->n_slots = static_cast<uint32_t>(cache->n_pages) << shift;
  out->page_shift = shift;
  out->H_kv = cfg->n_kv_heads;
  return SHOTKV_OK;
}

// Rows as the kernels take them: strides in bytes, every row 16-byte aligned.
int check_rows(const shotkv_config* cfg, const shotkv_rows* rows, RowView* out) {
  if (!rows || !rows->data) return SHOTKV_E_NULL;
  if (rows->seq_tokens < 1) return SHOTKV_E_SHAPE;
  const long long size = cfg->dtype == SHOTKV_BF16 ? 2 : 4;
  if (!aligned16(rows->data) || (rows->seq_stride * size) % 16 || (rows->token_stride * size) % 16 || (rows->head_stride * size) % 16)
    return SHOTKV_E_ALIGN;
  out->data = static_cast<char*>(rows->data);
  out->seq_stride = rows->seq_stride * size;
  out->token_stride = rows->token_stride * size;
  out->head_stride = rows->head_stride * size;
  out->seq_tokens = rows->seq_tokens;
  return SHOTKV_OK;
}

int from_hip(hipError_t e) { return e == hipSuccess ? SHOTKV_OK : SHOTKV_E_LAUNCH; }

int make_row_args(const shotkv_config* cfg, int T, const shotkv_rows* k, const shotkv_rows* v, const shotkv_kv4_cache* cache,
                  const int32_t* slot_map, Kv4RowArgs* a) {
  int rc = check_heads(cfg);
  if (rc != SHOTKV_OK) return rc;
  if (T < 0 || T > kMaxTokens) return SHOTKV_E_SHAPE;
  a->T = T;
  a->D = cfg->head_dim;
  a->dtype = cfg->dtype;
  a->slot_map = slot_map;
  if ((rc = check_cache(cfg, cache, &a->cache)) != SHOTKV_OK || T == 0) return rc;  // (no tokens, and there need be no arrays)
  if ((rc = check_rows(cfg, k, &a->k)) != SHOTKV_OK || (rc = check_rows(cfg, v, &a->v)) != SHOTKV_OK) return rc;
  return slot_map ? SHOTKV_OK : SHOTKV_E_NULL;
}

int make_attention_args(const shotkv_config* cfg, int R, int T, int max_q_len, int page_size, int max_pages, Kv4AttentionArgs* a) {
  const int rc = check_heads(cfg);
  if (rc != SHOTKV_OK) return rc;
  const int shift = log2_page(page_size);
  if (shift < 0 || R < 1 || R > kMaxRequests || T < 0 || T > kMaxTokens || max_q_len < 1 || max_q_len > kMaxTokens ||
      max_pages < 1 || static_cast<long long>(max_pages) << shift > kMaxLength)
    return SHOTKV_E_SHAPE;
  if (!(cfg->sm_scale > 0.f)) return SHOTKV_E_SHAPE;
  if (static_cast<long long>(max_q_len < T ? max_q_len : T) * cfg->n_q_heads > kMaxRows) return SHOTKV_E_SHAPE;
  *a = Kv4AttentionArgs{};
  a->R = R; a->T = T; a->H = cfg->n_q_heads; a->H_kv = cfg->n_kv_heads; a->G = a->H / a->H_kv; a->D = cfg->head_dim;
  a->dtype = cfg->dtype; a->max_q_len = max_q_len < T ? max_q_len : (T > 0 ? T : 1); a->max_pages = max_pages;
  a->sm_scale = cfg->sm_scale;
  a->cache.page_shift = shift;
  return SHOTKV_OK;
}

// Requests of up to kFewRows (token, head) rows per KV head are taken by one kernel, those of more by the other.  Where a
// call may hold both, both run, each past the requests of the other, unless the kernel for many would lose less by the short
// ones than the launches for few take, some 10 us: not above this many of their blocks for each of its workgroups.  In us with
// both kernels and with the one, 32 heads over 8, 128 channels, bf16: five chunks of 66 tokens and five single tokens of 375
// (1 block each) 41 and 32, a chunk of 100 and eight single tokens of 4096 (16) 58 and 53, sixteen of them (32) 65 and 74; in
// fp32, half as many workgroups, four of them (16) 71 and 69, eight (32) 75 and 96.
constexpr double kFewBlocks = 16;
bool may_be_few(const Kv4AttentionArgs& a) {
  const int few_tokens = kFewRows / a.G;
  // T tokens in R requests of up to max_q_len leave room for so many short ones
  const double left_out = static_cast<double>(a.R) * a.max_q_len - a.T;
  const double requests = fmin(left_out / (a.max_q_len - few_tokens), a.R - 1.0);
  const double blocks = static_cast<double>(static_cast<long long>(a.max_pages) << a.cache.page_shift) / kKv4Block;
  return few_tokens > 0 && requests * a.H_kv * blocks > kFewBlocks * many_rows_at_once(a);
}

struct AttentionPlan {
  bool few, many;
  TileShape few_shape, many_shape;
  size_t bytes;  // of the workspace
};
AttentionPlan plan_attention(const Kv4AttentionArgs& a) {
  AttentionPlan plan{};
  plan.many = static_cast<long long>(a.max_q_len) * a.G > kFewRows;
  plan.few = !plan.many || may_be_few(a);
  // sums, maxima and what is left of items: one launch after the other uses them
  auto need = [&](const TileShape& s) {
    const size_t rows = 2 * static_cast<size_t>(s.workgroups) * s.rows;
    return align_up(rows * a.D * 4, 256) + align_up(rows * 8, 256) + s.workgroups * sizeof(CutItem);
  };
  if (plan.few) plan.bytes = need(plan.few_shape = few_rows_shape(a));
  if (plan.many) {
    plan.many_shape = many_rows_shape(a);
    const size_t n = need(plan.many_shape);
    plan.bytes = n > plan.bytes ? n : plan.bytes;
  }
  plan.bytes = align_up(plan.bytes, 256);
  return plan;
}

hipError_t launch_attention(const Kv4AttentionArgs& a, void* workspace, hipStream_t s) {
  const AttentionPlan plan = plan_attention(a);
  AttnParams p{};
  p.R = a.R; p.T = a.T; p.H = a.H; p.H_kv = a.H_kv; p.G = a.G; p.max_q_len = a.max_q_len; p.max_pages = a.max_pages;
  p.scale_log2 = a.sm_scale * kLog2e;
  p.cache = a.cache;
  p.block_table = a.block_table; p.seq_lens = a.seq_lens; p.query_start = a.query_start;
  p.q = a.q; p.out = a.out; p.lse = a.lse;
  auto with = [&](const TileShape& shape, int least, int most) {
    AttnParams x = p;
    char* parts = static_cast<char*>(workspace);
    const size_t rows = 2 * static_cast<size_t>(shape.workgroups) * shape.rows;
    x.workgroups = shape.workgroups;
    x.least_rows = least;
    x.most_rows = most;
    x.part_o = reinterpret_cast<float*>(parts);
    x.part_ml = reinterpret_cast<float2*>(parts += align_up(rows * a.D * 4, 256));
    x.cut = reinterpret_cast<CutItem*>(parts + align_up(rows * 8, 256));
    return x;
  };
  if (plan.few) {
    const hipError_t e = launch_few_rows(with(plan.few_shape, 1, kFewRows), a.D, a.dtype, plan.few_shape.rows, s);
    if (e != hipSuccess) return e;
  }
  if (!plan.many) return hipSuccess;
  return launch_many_rows(with(plan.many_shape, plan.few ? kFewRows + 1 : 1, 0x7fffffff), a.D, a.dtype, s);
}

}  // namespace
}  // namespace shotkv

using namespace shotkv;

extern "C" {

size_t shotkv_kv4_page_bytes(int32_t page_size, int32_t n_kv_heads, int32_t head_dim) {
  if (log2_page(page_size) < 0 || n_kv_heads < 1 || n_kv_heads > 64 || (head_dim != 64 && head_dim != 128)) return 0;
  return kv4_page_bytes(page_size, n_kv_heads, head_dim);
}

int shotkv_pages_plan(int32_t R, int32_t page_size, int32_t max_pages, const int32_t* cached_lens, const int32_t* new_lens,
                      const int32_t* pos_start, const int32_t* free_pages, int32_t stack_size, const int32_t* free_count,
                      int32_t* block_table, int32_t* free_left, int32_t* seq_lens, int32_t* query_start, int32_t T,
                      int32_t request_tokens, int32_t* slot_map, int32_t* token_pos, int32_t* status, void* stream) {
  const int shift = log2_page(page_size);
  if (shift < 0 || R < 1 || R > kMaxRequests || max_pages < 1 || static_cast<long long>(max_pages) << shift > kMaxLength ||
      stack_size < 0 || T < 0 || T > kMaxTokens || request_tokens < 0)
    return SHOTKV_E_SHAPE;
  if (!cached_lens || !new_lens || (!free_pages && stack_size > 0) || !free_count || !block_table || !free_left || !seq_lens || !query_start ||
      !status || (T > 0 && (!slot_map || !token_pos)))
    return SHOTKV_E_NULL;
  if (free_left == free_count || seq_lens == cached_lens) return SHOTKV_E_SHAPE;  // others still read what one would write
  return from_hip(launch_pages_plan(R, shift, max_pages, cached_lens, new_lens, pos_start, free_pages, stack_size, free_count,
                                    block_table, free_left, seq_lens, query_start, T, request_tokens, slot_map, token_pos, status,
                                    static_cast<hipStream_t>(stream)));
}

int shotkv_pages_release(int32_t R, int32_t page_size, int32_t max_pages, const uint8_t* finished, int32_t* seq_lens,
                         int32_t* block_table, int32_t* free_pages, int32_t stack_size, int32_t* free_count, void* stream) {
  const int shift = log2_page(page_size);
  if (shift < 0 || R < 1 || R > kMaxRequests || max_pages < 1 || static_cast<long long>(max_pages) << shift > kMaxLength ||
      stack_size < 0)
    return SHOTKV_E_SHAPE;
  if (!finished || !seq_lens || !block_table || !free_pages || !free_count) return SHOTKV_E_NULL;
  return from_hip(launch_pages_release(R, shift, max_pages, finished, seq_lens, block_table, free_pages, stack_size, free_count,
                                       static_cast<hipStream_t>(stream)));
}

int shotkv_qk_norm_rope(const shotkv_config* cfg, int32_t T, const shotkv_rope* rope, const int32_t* token_pos,
                        const shotkv_rows* q, const shotkv_rows* k, const shotkv_rows* q_out, const shotkv_rows* k_out,
                        const shotkv_rows* v, const shotkv_kv4_cache* cache, const int32_t* slot_map, void* stream) {
  int rc = check_heads(cfg);
  if (rc != SHOTKV_OK) return rc;
  if (T < 0 || T > kMaxTokens) return SHOTKV_E_SHAPE;
  if (!rope || (T > 0 && !token_pos)) return SHOTKV_E_NULL;
  if (rope->rot_dim < 16 || rope->rot_dim % 16 || rope->rot_dim > cfg->head_dim || rope->n_positions < 1 || !(rope->eps >= 0.f))
    return SHOTKV_E_SHAPE;
  if (!rope->table) return SHOTKV_E_NULL;
  if (!aligned16(rope->table) || !aligned16(rope->q_weight) || !aligned16(rope->k_weight)) return SHOTKV_E_ALIGN;
  if (T == 0) return SHOTKV_OK;
  const bool stores = cache || v || slot_map;
  if (stores && (!cache || !v || !slot_map)) return SHOTKV_E_NULL;
  if (!stores && !k_out) return SHOTKV_E_NULL;
  RopeArgs a{};
  a.T = T; a.H = cfg->n_q_heads; a.H_kv = cfg->n_kv_heads; a.D = cfg->head_dim; a.dtype = cfg->dtype;
  a.table = rope->table; a.n_positions = rope->n_positions; a.rot_dim = rope->rot_dim; a.interleaved = rope->interleaved != 0;
  a.eps = rope->eps; a.q_weight = rope->q_weight; a.k_weight = rope->k_weight;
  a.token_pos = token_pos; a.slot_map = slot_map;
  if ((rc = check_rows(cfg, q, &a.q)) != SHOTKV_OK || (rc = check_rows(cfg, k, &a.k)) != SHOTKV_OK ||
      (rc = check_rows(cfg, q_out, &a.q_out)) != SHOTKV_OK)
    return rc;
  if (k_out && (rc = check_rows(cfg, k_out, &a.k_out)) != SHOTKV_OK) return rc;
  if (stores && ((rc = check_rows(cfg, v, &a.v)) != SHOTKV_OK || (rc = check_cache(cfg, cache, &a.cache)) != SHOTKV_OK)) return rc;
  return from_hip(launch_norm_rope(a, static_cast<hipStream_t>(stream)));
}

int shotkv_kv4_store(const shotkv_config* cfg, int32_t T, const shotkv_rows* k, const shotkv_rows* v,
                     const shotkv_kv4_cache* cache, const int32_t* slot_map, void* stream) {
  Kv4RowArgs a{};
  const int rc = make_row_args(cfg, T, k, v, cache, slot_map, &a);
  if (rc != SHOTKV_OK || T == 0) return rc;
  return from_hip(launch_kv4_store(a, static_cast<hipStream_t>(stream)));
}

int shotkv_kv4_load(const shotkv_config* cfg, int32_t T, const shotkv_kv4_cache* cache, const int32_t* slot_map,
                    const shotkv_rows* k, const shotkv_rows* v, void* stream) {
  Kv4RowArgs a{};
  const int rc = make_row_args(cfg, T, k, v, cache, slot_map, &a);
  if (rc != SHOTKV_OK || T == 0) return rc;
  return from_hip(launch_kv4_load(a, static_cast<hipStream_t>(stream)));
}

size_t shotkv_kv4_attention_workspace_bytes(const shotkv_config* cfg, int32_t R, int32_t T, int32_t max_q_len, int32_t page_size,
                                            int32_t max_pages) {
  Kv4AttentionArgs a;
  if (make_attention_args(cfg, R, T, max_q_len, page_size, max_pages, &a) != SHOTKV_OK) return 0;
  return plan_attention(a).bytes;
}

int shotkv_kv4_attention(const shotkv_config* cfg, int32_t R, int32_t T, int32_t max_q_len, const shotkv_kv4_cache* cache,
                         const int32_t* block_table, int32_t max_pages, const int32_t* seq_lens, const int32_t* query_start,
                         const shotkv_rows* q, const shotkv_rows* out, float* lse, void* workspace, size_t workspace_bytes,
                         void* stream) {
  if (!cache) return SHOTKV_E_NULL;
  Kv4AttentionArgs a;
  int rc = make_attention_args(cfg, R, T, max_q_len, cache->page_size, max_pages, &a);
  if (rc != SHOTKV_OK) return rc;
  if (!query_start && T != R) return SHOTKV_E_SHAPE;
  if (!block_table || !seq_lens || !workspace) return SHOTKV_E_NULL;
  if ((rc = check_cache(cfg, cache, &a.cache)) != SHOTKV_OK || T == 0) return rc;
  if ((rc = check_rows(cfg, q, &a.q)) != SHOTKV_OK ||
      (rc = check_rows(cfg, out, &a.out)) != SHOTKV_OK)
    return rc;
  if (!aligned16(workspace)) return SHOTKV_E_ALIGN;
  if (workspace_bytes < plan_attention(a).bytes) return SHOTKV_E_WORKSPACE;
  a.block_table = block_table; a.seq_lens = seq_lens; a.query_start = query_start; a.lse = lse;
  return from_hip(launch_attention(a, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
