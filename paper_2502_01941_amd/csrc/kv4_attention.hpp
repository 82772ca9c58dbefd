// What the two attention kernels over the paged 4-bit cache share: requests, the division of work, the rows' output.
//
// Work is cut by blocks of 32 tokens, not by requests.  An item is a tile of query rows of one (request, KV head), as long as
// its visible blocks; all items in a row, with a constant for each one's start, are shared equally by the workgroups, whatever
// the lengths.  An item that one workgroup has to itself is finished there; of the others the workgroups leave parts (maximum,
// sum of weights, weighted sum of values), which a second kernel joins.
#pragma once

#include "kv4.hpp"

namespace shotkv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(2))) float floatx2;

constexpr int kCus = 256;
// A running maximum before any key that the row sees, and of a row all of whose keys so far have logits of -infinity: below all
// others and finite, so that no difference of two of them is NaN.
constexpr float kLowest = -3.402823466e38f, kNoFinite = -3.402823264e38f;
// The softmax reference is a running maximum that is let fall behind by up to this much (log2): weights of up to 2^8 are as
// exact in bf16 and in 32-bit sums as those up to 1, and most blocks need neither the maximum over lanes nor new sums.
constexpr float kSlack = 8.f;
constexpr float kLn2 = 0.6931471805599453f;
// Weights are 2^(by * logit - reference), in one rounding, of a reference that is by * (largest logit), rounded: off by up to
// 2^-24 of it, a factor of 2^that in all weights of the row, which cancels as long as 32-bit numbers hold it.  References above
// 2^28 are therefore made exact: `by` is there the power of two next below sm_scale * log2(e).  (Logits of that size are at least
// 16 apart, or equal, and themselves rounded to such steps: other weights than those of the largest are next to none either way.)
// Rounding every logit by itself in rows of that size, by a branch in every block, took 825 us where this takes 735 (4 x 1024 new
// tokens of 4096, fp32; 707 without either).
constexpr float kLarge = 268435456.f;
struct Reference {
  float m, by;
  // Takes the row's largest logit of a block into account; the factor that sums so far are to be taken by.
  __device__ __forceinline__ float raise(float logit, float scale_log2) {
    const float grown = logit * by;
    if (!(grown > m)) return 1.f;
    const float shrink = __builtin_amdgcn_exp2f(m - grown);
    by = fabsf(logit * scale_log2) > kLarge ? __uint_as_float(__float_as_uint(scale_log2) & 0x7f800000u) : scale_log2;
    m = logit * by;
    return shrink;
  }
  // The reference with by = scale_log2, as the sums' is at the end.
  __device__ __forceinline__ float scaled(float scale_log2) const {
    return by == scale_log2 ? m : fmaxf(m * (scale_log2 / by), kNoFinite);
  }
};

// The item that a workgroup begins and leaves to the ones after it: all that the join has to know of it.
struct alignas(32) CutItem {
  int first_row, head, tile;  // its request's first token in the batch
  int rows;                   // of the tile; 0: the workgroup leaves none
  int last;                   // workgroup that ends it
};

struct AttnParams {
  int R, T, H, H_kv, G, max_q_len, max_pages, workgroups;
  int least_rows, most_rows;  // (token, head) rows of the requests that a launch takes; others are not there for it
  float scale_log2;
  Kv4Pages cache;
  const int32_t *block_table, *seq_lens, *query_start;
  RowView q, out;
  float* lse;
  CutItem* cut;     // [workgroups]
  float2* part_ml;  // [2 * workgroups][rows of a tile]: maximum, sum
  float* part_o;    // [2 * workgroups][rows of a tile][D]
};

struct Request {
  int first_row;  // of its tokens in the batch
  int q_len, len; // new tokens that the launch takes; cached tokens up to the last of them (below 0: that many see nothing)
  __device__ __forceinline__ Request of_lane(int lane) const {
    return {__builtin_amdgcn_readlane(first_row, lane), __builtin_amdgcn_readlane(q_len, lane), __builtin_amdgcn_readlane(len, lane)};
  }
};

__device__ __forceinline__ Request request_of(const AttnParams& p, int r) {
  Request q;
  const long long most = static_cast<long long>(p.max_pages) << p.cache.page_shift;
  q.len = static_cast<int>(min(static_cast<long long>(max(p.seq_lens[r], 0)), most));
  if (p.query_start) {
    const int first = min(max(p.query_start[r], 0), p.T), end = min(max(p.query_start[r + 1], 0), p.T);
    const int fresh = max(end - first, 0);
    q.first_row = first;
    q.q_len = min(fresh, p.max_q_len);
    q.len -= fresh - q.q_len;  // with the tokens that are cut off go the keys that only those see
  } else {
    q.first_row = r;
    q.q_len = 1;
  }
  const int rows = q.q_len * p.G;
  if (rows < p.least_rows || rows > p.most_rows) q.q_len = 0;
  return q;
}

// Keys that the tokens up to token i of a request see.
__device__ __forceinline__ int visible(const Request& q, int i) { return max(q.len - q.q_len + i + 1, 0); }

// The constants of a kernel: rows of a tile, the units that an item's start counts for (its queries, its first trips to
// memory and its end take as long as that many blocks), the least units of a workgroup.
template <int ROWS, int ITEM_UNITS, int MIN_UNITS>
struct Division {
  static constexpr int kRows = ROWS, kItemUnits = ITEM_UNITS, kMinUnits = MIN_UNITS;
  static __device__ __forceinline__ int tiles(const Request& q, int G) { return (q.q_len * G + ROWS - 1) / ROWS; }
  // Blocks that a tile of rows goes through; a tile whose rows see nothing has one, of which it sees nothing.
  static __device__ __forceinline__ int blocks(const Request& q, int G, int tile) {
    const int last = min(static_cast<int>(static_cast<uint32_t>(tile * ROWS + ROWS - 1) / static_cast<uint32_t>(G)), q.q_len - 1);
    return max((visible(q, last) + kKv4Block - 1) / kKv4Block, 1);
  }
  // Units of the tiles [from, to), every `step`th.
  static __device__ __forceinline__ long long units(const Request& q, int G, int from, int to, int step = 1) {
    long long sum = 0;
    for (int t = from; t < to; t += step) sum += blocks(q, G, t) + kItemUnits;
    return sum;
  }
  // Units of a workgroup: `workgroups` times as many are all of them.
  static __device__ __forceinline__ long long share(long long total, int workgroups);
};

// a / b of numbers below 2^52, a >= 0, b > 0, by an estimate and exact corrections.
__device__ __forceinline__ long long quotient(long long a, long long b) {
  if (a < (1ll << 30) && b < (1ll << 30)) {
    const int x = static_cast<int>(a), y = static_cast<int>(b);
    const float inverse = __builtin_amdgcn_rcpf(static_cast<float>(y));
    int q = static_cast<int>(static_cast<float>(x) * inverse);            // 2^-21 of it off
    q += static_cast<int>(floorf(static_cast<float>(x - q * y) * inverse));  // 1 off
    const int rest = x - q * y;
    return rest < 0 ? q - 1 : rest >= y ? q + 1 : q;
  }
  const long long q = static_cast<long long>(static_cast<double>(a) / static_cast<double>(b));
  const long long rest = a - q * b;
  return rest < 0 ? q - 1 : rest >= b ? q + 1 : q;
}
template <int ROWS, int ITEM_UNITS, int MIN_UNITS>
__device__ __forceinline__ long long Division<ROWS, ITEM_UNITS, MIN_UNITS>::share(long long total, int workgroups) {
  return max(quotient(total + workgroups - 1, workgroups), static_cast<long long>(MIN_UNITS));
}
__device__ __forceinline__ long long read_lane64(long long v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), lane);
  return static_cast<long long>(static_cast<unsigned long long>(hi) << 32 | lo);
}
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ uint32_t add_shifted(uint32_t v) {
  return v + __builtin_amdgcn_update_dpp(0u, v, CTRL, ROW_MASK, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_scan32(uint32_t v) {
  v = add_shifted<0x111, 0xf>(v);  // row_shr:1, 2, 4, 8: sums within 16 lanes
  v = add_shifted<0x112, 0xf>(v);
  v = add_shifted<0x114, 0xf>(v);
  v = add_shifted<0x118, 0xf>(v);
  v = add_shifted<0x142, 0xa>(v);  // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
  return add_shifted<0x143, 0xc>(v);
}
// Sum up to and with this lane, of numbers below 2^48.
__device__ __forceinline__ long long wave_scan(long long v) {
  const uint32_t low = wave_scan32(static_cast<uint32_t>(v) & 0xffffffu), high = wave_scan32(static_cast<uint32_t>(v >> 24));
  return (static_cast<long long>(high) << 24) + low;
}
// Sum over the threads before this one; *total grows by the sum over all.
template <int WAVES>
__device__ __forceinline__ long long block_scan(long long v, int lane, int wave, long long* scratch, long long* total) {
  const long long sum = wave_scan(v);
  __syncthreads();
  if (lane == kWave - 1) scratch[wave] = sum;
  __syncthreads();
  long long before = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    if (i < wave) before += scratch[i];
    *total += scratch[i];
  }
  return before + sum - v;
}

template <int I>
struct Constant {
  static constexpr int value = I;
};

__device__ __forceinline__ bf16x8 words_to_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8, (u32x4{a, b, c, d}));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{a, b}), bf16x2));
}
// x - the low (by = (-1, 0)) or the high (0, -1) half of w, or x (0, 0): exact, in one instruction.
__device__ __forceinline__ float less(float x, uint32_t w, uint32_t by) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, by), x, false);
}
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// An output row: row `flat` of the (token, head of the group) rows of the request whose first token is first_row, from its
// maximum and sums.
template <typename T>
struct RowOut {
  char* dst;
  float* lse;
  float inv, top, sum;
  __device__ __forceinline__ RowOut(const AttnParams& p, int first_row, int head, int flat, float top_, float sum_) : top(top_), sum(sum_) {
    const int token = flat / p.G, h = head * p.G + flat - token * p.G;
    dst = p.out.token(first_row + token) + h * p.out.head_stride;
    lse = p.lse ? p.lse + static_cast<size_t>(first_row + token) * p.H + h : nullptr;
    // no weight: a row that sees no key, or one whose logits are all -infinity
    inv = sum != 0.f ? 1.f / sum : top > kLowest ? NAN : 0.f;
  }
  __device__ __forceinline__ void write(int ch, const float4& x) const {  // four channels from ch on
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x2*>(dst + ch * 2) = u32x2{pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv)};
    } else {
      *reinterpret_cast<float4*>(dst + ch * 4) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    }
  }
  __device__ __forceinline__ void write_lse() const {
    if (lse) *lse = sum != 0.f ? add_log2(top, sum) * kLn2 : top > kLowest ? NAN : -INFINITY;
  }
};

// The reference that a row passes on whose last visible key is `last`, after the blocks from, from + step, ... before `end`.  Where
// it is the lowest still, whether the row saw a key at all is looked up in the table.
__device__ __forceinline__ float passed_on(const AttnParams& p, const Reference& ref, int last, const int32_t* table, int from, int step, int end) {
  const float m = ref.scaled(p.scale_log2);
  if (m == kLowest)
    for (int b = from; b < end && b * kKv4Block <= last; b += step) {
      const int page = table[min(b >> (p.cache.page_shift - 5), p.max_pages - 1)];
      if (page >= 0 && page < p.cache.n_pages) return kNoFinite;
    }
  return m;
}

// What workgroup `workgroup` begins and does not end: an item whose last unit is last_unit.
__device__ __forceinline__ void leave_item(const AttnParams& p, int workgroup, const Request& rq, int head, int tile, int rows,
                                           long long last_unit, long long share) {
  if (threadIdx.x == 0)
    p.cut[workgroup] = CutItem{rq.first_row, head, tile, rows, static_cast<int>(quotient(last_unit, share))};
}

// Sum over a workgroup of THREADS threads; every thread gets it.
template <int THREADS>
__device__ __forceinline__ long long block_sum(long long v, long long* scratch) {
  v = read_lane64(wave_scan(v), kWave - 1);
  __syncthreads();
  if (threadIdx.x % kWave == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  long long sum = 0;
#pragma unroll
  for (int i = 0; i < THREADS / kWave; ++i) sum += scratch[i];
  return sum;
}

// Joins the parts of the items that several workgroups shared: workgroup (workgroup that begins an item, slice of its rows).
// The threads of a row's four channels share its parts, four of them in flight each, every thread with a maximum of its own.
constexpr int kJoinRows = 8;  // of a slice
// The fewer rows, the more parts an item has and the fewer workgroups.  Single tokens: 1024 threads 3.2 us, 512 3.8 (one
// request of 3277 tokens, 15 parts to a head); tiles of 128 rows: 256 threads 15.5 us, 512 17.8, 1024 32 (2048 new tokens of
// 32768, two or three parts to a tile).
constexpr int join_threads(int rows) { return rows <= 8 ? 1024 : rows <= 32 ? 512 : 256; }
template <int D, typename T, int ROWS>
__global__ __launch_bounds__(join_threads(ROWS)) void kv4_join_kernel(AttnParams p) {
  constexpr int kThreads = join_threads(ROWS);
  constexpr int kCells = kJoinRows * (D / 4), kShares = kThreads / kCells;
  const CutItem item = p.cut[blockIdx.x];
  if (static_cast<int>(blockIdx.y) * kJoinRows >= item.rows) return;
  const int w0 = blockIdx.x, w1 = item.last;
  const int cell = threadIdx.x % kCells, row = blockIdx.y * kJoinRows + cell / (D / 4), ch = cell % (D / 4) * 4;
  float top = kLowest, sum = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  if (row < item.rows) {
    constexpr int kDeep = 4;
    for (int w = w0 + threadIdx.x / kCells; w <= w1; w += kShares * kDeep) {
      float2 ml[kDeep];
      float4 y[kDeep];
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        const int wi = min(w + i * kShares, w1);
        // the first part is the one that begins the item, the others are their workgroups' first
        const size_t part = 2 * static_cast<size_t>(wi) + (wi == w0 ? 1 : 0);
        ml[i] = p.part_ml[part * ROWS + row];
        y[i] = *reinterpret_cast<const float4*>(p.part_o + (part * ROWS + row) * D + ch);
      }
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        if (w + i * kShares > w1) continue;
        const float grown = fmaxf(top, ml[i].x), f = __builtin_amdgcn_exp2f(top - grown), g = __builtin_amdgcn_exp2f(ml[i].x - grown);
        x.x = x.x * f + y[i].x * g; x.y = x.y * f + y[i].y * g; x.z = x.z * f + y[i].z * g; x.w = x.w * f + y[i].w * g;
        sum = sum * f + ml[i].y * g;
        top = grown;
      }
    }
  }
  if constexpr (kShares > 1) {
    __shared__ __align__(16) float4 sh_x[kThreads];
    __shared__ float2 sh_ml[kThreads];
    sh_x[threadIdx.x] = x;
    sh_ml[threadIdx.x] = make_float2(top, sum);
    __syncthreads();
    if (threadIdx.x >= kCells) return;
#pragma unroll
    for (int i = 1; i < kShares; ++i) {
      const float2 ml = sh_ml[cell + i * kCells];
      const float4 y = sh_x[cell + i * kCells];
      const float grown = fmaxf(top, ml.x), f = __builtin_amdgcn_exp2f(top - grown), g = __builtin_amdgcn_exp2f(ml.x - grown);
      x.x = x.x * f + y.x * g; x.y = x.y * f + y.y * g; x.z = x.z * f + y.z * g; x.w = x.w * f + y.w * g;
      sum = sum * f + ml.y * g;
      top = grown;
    }
  }
  if (row >= item.rows) return;
  const RowOut<T> out(p, item.first_row, item.head, item.tile * ROWS + row, top, sum);
  out.write(ch, x);
  if (ch == 0) out.write_lse();
}
template <int D, typename T, int ROWS>
hipError_t launch_join(const AttnParams& p, hipStream_t s) {
  kv4_join_kernel<D, T, ROWS><<<dim3(p.workgroups - 1, ROWS / kJoinRows), join_threads(ROWS), 0, s>>>(p);  // the last leaves none
  return hipGetLastError();
}

// (token, head) rows per KV head up to which requests are taken by the kernel for few rows.  At 32 rows (16 requests of 4096, 8
// new tokens, 128 channels) it takes 33.6 us and the other 40, in fp32 44 and 72, of 64 channels 27 and 31, in fp32 30 and 36; at
// 48 it would go over the cache twice, the other takes 49.
constexpr int kFewRows = 32;
// Launches of the two kernels and what they need: tiles of so many rows, so many workgroups.
struct TileShape {
  int rows, workgroups;
};
TileShape few_rows_shape(const Kv4AttentionArgs& a);
hipError_t launch_few_rows(const AttnParams& p, int D, int dtype, int rows, hipStream_t s);
TileShape many_rows_shape(const Kv4AttentionArgs& a);
int many_rows_at_once(const Kv4AttentionArgs& a);  // workgroups
hipError_t launch_many_rows(const AttnParams& p, int D, int dtype, hipStream_t s);

}  // namespace shotkv
