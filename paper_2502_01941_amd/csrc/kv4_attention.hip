// Attention of a few query rows per KV head over the paged 4-bit cache: single tokens, drafts, and (as tiles of rows) any
// number of new tokens.
//
// Per request and KV head: S^T = K Q^T, weights 2^(S - m), O^T += V^T P^T over the cached tokens in blocks of 32, with the
// running maximum m and sum of a softmax that is computed in one pass.  v_mfma_f32_16x16x32_bf16 makes both products; codes
// times a power of two are exact in bf16, so keys and values enter them as the cache holds them.
//   keys      A rows are 16 tokens; lane (token, kg) holds the codes of one group of 32 channels (D = 128) with its one
//             scale, 16 bytes in one load, and word j of it is its share of step j: channels 32 kg + 8 j ..+7.  Queries are
//             laid out to match, so no lane exchanges anything.
//   weights   what a lane holds of S^T after the softmax (columns are query rows) is the B operand of the second product,
//             if that takes its 32 tokens in the order {4 kg + i, 16 + 4 kg + i}.
//   values    lane (chunk of 8 channels, kg) loads four tokens' words of one chunk as 16 bytes, twice: the same tokens.
//             Converted, pairs of tokens are put together per channel, which makes the A operand for eight times 16 channels.
// Nothing goes through LDS until the four waves of a workgroup, which take blocks in turn, join their sums at the end.
//
// Precision: sums, maxima and the output are 32-bit.  A weight is the sum of two bf16 numbers (2^-16 off at most; as one it
// would be off by up to 2^-8, as much as a bf16 output's own rounding), of three where the output is fp32: what the first
// leaves goes through the second product once more.  Up to eight rows leave half of the columns empty; there columns 8..15
// repeat the query rows of columns 0..7 and hold the second numbers (PAIRED), at no further matrix work.  fp32 queries are
// the sum of three bf16 numbers, in three products.
//
// Work is cut by blocks, not by requests: all (request, KV head, tile of rows) items in a row, each as long as its visible
// blocks, are shared equally by the workgroups, whatever the lengths.  An item that one workgroup has to itself is finished
// there; the parts of the others are joined by a second kernel.
#include "kv4.hpp"

namespace shotkv {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(2))) float floatx2;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kRingBlocks = 3;
constexpr int kCus = 256;
constexpr int kMinUnits = 8;          // of a workgroup: two blocks to a wave
constexpr int kItemUnits = 16;
constexpr float kLowest = -1e30f;     // a running maximum before any key
// The softmax reference is a running maximum that is let fall behind by up to this much (log2): weights of up to 2^8 are as
// exact in bf16 and in 32-bit sums as those up to 1, and most blocks need neither the maximum over lanes nor new sums.
constexpr float kSlack = 8.f;
constexpr float kLn2 = 0.6931471805599453f;

struct Params {
  int R, T, H, H_kv, G, max_q_len, max_pages, workgroups;
  float scale_log2;
  Kv4Pages cache;
  const int32_t *block_table, *seq_lens, *query_start;
  RowView q, out;
  float* lse;
  long long* first_unit;  // [R + 1] units before each request
  float2* part_ml;         // [2 * workgroups][rows]
  float* part_o;           // [2 * workgroups][rows][D]
};

struct Request {
  int first_row;  // of its tokens in the batch
  int q_len, len;
};

__device__ __forceinline__ Request request_of(const Params& p, int r) {
  Request q;
  const long long most = static_cast<long long>(p.max_pages) << p.cache.page_shift;
  q.len = static_cast<int>(min(static_cast<long long>(max(p.seq_lens[r], 0)), most));
  if (p.query_start) {
    q.first_row = min(max(p.query_start[r], 0), p.T);
    q.q_len = min(min(max(p.query_start[r + 1] - q.first_row, 0), p.max_q_len), p.T - q.first_row);
  } else {
    q.first_row = r;
    q.q_len = 1;
  }
  return q;
}

// Keys that the tokens up to token i of a request see.
__device__ __forceinline__ int visible(const Request& q, int i) { return max(q.len - q.q_len + i + 1, 0); }

template <int ROWS>
__device__ __forceinline__ int tiles_of(const Request& q, int G) { return (q.q_len * G + ROWS - 1) / ROWS; }
// Blocks that a tile of rows goes through; a tile whose rows see nothing has one, of which it sees nothing.
template <int ROWS>
__device__ __forceinline__ int blocks_of(const Request& q, int G, int tile) {
  const int last = min((tile * ROWS + ROWS - 1) / G, q.q_len - 1);
  return max((visible(q, last) + kKv4Block - 1) / kKv4Block, 1);
}
// What an item counts for: its blocks, and for its queries, its first trips to memory and the join of its waves as many
// again as pass in that time.
template <int ROWS>
__device__ __forceinline__ long long units_of_head(const Request& q, int G) {
  const int tiles = tiles_of<ROWS>(q, G);
  long long sum = static_cast<long long>(tiles) * kItemUnits;
  for (int t = 0; t < tiles; ++t) sum += blocks_of<ROWS>(q, G, t);
  return sum;
}

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
// Units of a workgroup: `workgroups` times as many are all of them.
__device__ __forceinline__ long long share_of(long long total, int workgroups) {
  return max(quotient(total + workgroups - 1, workgroups), static_cast<long long>(kMinUnits));
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
__device__ __forceinline__ long long block_scan(long long v, int lane, int wave, long long* scratch, long long* total) {
  const long long sum = wave_scan(v);
  __syncthreads();
  if (lane == kWave - 1) scratch[wave] = sum;
  __syncthreads();
  long long before = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) before += scratch[i];
    *total += scratch[i];
  }
  return before + sum - v;
}

// Blocks on their way: every wave has a ring of them in LDS that it fills and reads by itself, straight from memory
// (global_load_lds: lane l's 16 bytes go to 16 l), so what is in flight takes no registers and waits for nobody.  Keys of 128
// channels are fetched so that lane l finds its codes at 16 l as well.
template <int D>
struct Ring {
  static constexpr int kSlot = 32 * D + 256;  // codes, and the scales (of 128 bytes in D = 64, twice)
  static constexpr int kDepth = kRingBlocks;
  static constexpr int kBytes = kWaves * kDepth * kSlot;
  static constexpr int kLoads = D == 128 ? 5 : 3;  // instructions of a block
};

// The slot has the block's own layout (an instruction's offset counts in memory and in LDS).
template <int D>
__device__ __forceinline__ void request_block(const char* base, uint32_t slot, uint32_t key_piece, uint32_t straight, uint32_t word) {
  if constexpr (D == 128) {
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %2, %5 nt\n\tglobal_load_lds_dwordx4 %2, %5 offset:1024 nt\n\t"
        "global_load_lds_dwordx4 %3, %5 offset:2048 nt\n\tglobal_load_lds_dwordx4 %3, %5 offset:3072 nt\n\t"
        "s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %4, %5 nt"
        :
        : "s"(slot), "s"(slot + 4096), "v"(key_piece), "v"(straight), "v"(word), "s"(base)
        : "memory", "m0");
  } else {
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %3 nt\n\tglobal_load_lds_dwordx4 %1, %3 offset:1024 nt\n\t"
        "global_load_lds_dword %2, %3 offset:2048 nt"
        :
        : "s"(slot), "v"(straight), "v"(word), "s"(base)
        : "memory", "m0");
  }
}
// All but the youngest `blocks` blocks have arrived.
template <int D>
__device__ __forceinline__ void wait_block(int blocks) {
  constexpr int n = Ring<D>::kLoads;
  if (blocks >= 3) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(3 * n) : "memory");
  else if (blocks == 2) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * n) : "memory");
  else if (blocks == 1) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(n) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
}

// What a lane takes of a block.
template <int D>
struct BlockData {
  uint32_t k[2][D / 32];  // two times 16 tokens: this lane's share of its token
  uint32_t ks[2];
  u32x4 v[2];             // two quads of tokens: this lane's chunk of channels
  uint32_t vs[2];
};
typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) const u32x2 lds_u32x2;
typedef __attribute__((address_space(3))) const uint32_t lds_u32;
typedef __attribute__((address_space(3))) const uint8_t lds_u8;
template <int D>
__device__ __forceinline__ void read_block(uint32_t slot, int lane, BlockData<D>& b) {
  const int c = lane & 15, kg = lane >> 4, chunk = c % (D / 8);
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    if constexpr (D == 128) {
      const u32x4 w = *reinterpret_cast<lds_u32x4*>(static_cast<uintptr_t>(slot + a * 1024 + lane * 16));
#pragma unroll
      for (int j = 0; j < 4; ++j) b.k[a][j] = w[j];
    } else {
      const u32x2 w = *reinterpret_cast<lds_u32x2*>(static_cast<uintptr_t>(slot + a * 512 + c * 32 + kg * 8));
      b.k[a][0] = w[0];
      b.k[a][1] = w[1];
    }
    const int quad = a * 4 + kg;
    b.ks[a] = *reinterpret_cast<lds_u8*>(static_cast<uintptr_t>(slot + 32 * D + (a * 16 + c) * (D / 32) + kg * (D / 32) / 4));
    b.v[a] = *reinterpret_cast<lds_u32x4*>(static_cast<uintptr_t>(slot + 16 * D + (quad * (D / 8) + chunk) * 16));
    b.vs[a] = *reinterpret_cast<lds_u32*>(static_cast<uintptr_t>(slot + 33 * D + (quad * (D / 32) + chunk / 4) * 4));
  }
}

template <int I>
struct Constant {
  static constexpr int value = I;
};

__device__ __forceinline__ bf16x8 words_to_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8, (u32x4{a, b, c, d}));
}
__device__ __forceinline__ bf16x8 decode_word(uint32_t codes, float scale) {
  return words_to_bf16x8(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)));
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

__device__ __forceinline__ float max_across_rows(float x) {  // over lanes 16, 32 and 48 away
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_across_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_across_rows(float x) { return sum_across_halves(sum_across_row_pairs(x)); }

// Four channels of an output row: row `flat` of the request's (token, head of the group) rows.
template <typename T>
__device__ __forceinline__ void write_row(const Params& p, const Request& rq, int head, int flat, int ch, const float4& x, float top,
                                          float sum) {
  const int token = flat / p.G, h = flat - token * p.G;
  const float inv = sum != 0.f ? 1.f / sum : 0.f;
  char* dst = p.out.token(rq.first_row + token) + (head * p.G + h) * p.out.head_stride;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x2*>(dst + ch * 2) = u32x2{pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv)};
  } else {
    *reinterpret_cast<float4*>(dst + ch * 4) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
  }
  if (ch == 0 && p.lse)
    p.lse[static_cast<size_t>(rq.first_row + token) * p.H + head * p.G + h] = sum != 0.f ? add_log2(top, sum) * kLn2 : -INFINITY;
}

// Workgroups of a CU at once: four waves each, of up to 168 registers in the form for single tokens in bf16, of up to 256 in
// the others.
constexpr int workgroups_per_cu(bool f32, int rows) { return f32 || rows > 16 ? 2 : 3; }

// T: storage type of queries and output.  COLS: query rows of a set of 16 columns (8 if PAIRED).  NC: sets of columns.
template <int D, typename T, int NC, bool PAIRED>
__global__ __launch_bounds__(kThreads, workgroups_per_cu(sizeof(T) == 4, (PAIRED ? 8 : 16) * NC)) void kv4_attention_kernel(Params p) {
  constexpr int COLS = PAIRED ? 8 : 16, ROWS = COLS * NC;
  constexpr int kSteps = D / 32;                    // of the first product
  constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;    // bf16 numbers that a query element is the sum of
  constexpr int kNumbers = sizeof(T) == 4 ? 3 : 2;  // bf16 numbers that a weight is the sum of
  constexpr int kParts = PAIRED ? kNumbers - 1 : kNumbers;  // products that a weight goes through
  constexpr int kFrags = D / 16;                    // 16 channels each of the second product
  constexpr int kPad = D + 4;
  __shared__ long long scan[kWaves + 1];
  __shared__ long long found[2];
  __shared__ float sh_m[kWaves][ROWS], sh_l[kWaves][ROWS];
  typedef Ring<D> R;
  constexpr int kSums = kWaves * ROWS * kPad * 4;
  __shared__ __align__(16) char lds[kSums > R::kBytes ? kSums : R::kBytes];  // the rings, and then the waves' sums
  float (*sh_o)[ROWS][kPad] = reinterpret_cast<float (*)[ROWS][kPad]>(lds);
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = lane & 15, kg = lane >> 4;

  const uint32_t ring = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds)) + wave * R::kDepth * R::kSlot;

  const bf16x8 ones = words_to_bf16x8(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
  uint32_t low = 0x0000bf80u, high = 0xbf800000u;
  asm("" : "+s"(low), "+s"(high));  // (as known constants they would become the inline -1.0, which is the high half for both)
  const uint32_t upper_low = c < 8 ? 0u : low, upper_high = c < 8 ? 0u : high;
  // where this lane fetches from in a block: keys, values, scales
  const uint32_t straight = lane * 16, key_piece = c * 64 + kg * 16, word = D == 128 ? 4096 + lane * 4 : (lane & 31) * 4;

  // ---- this workgroup's share of the blocks, and the request that holds its first
  long long at, end, rest;
  int r;
  auto work_of = [&](int i) -> long long { return i < p.R ? units_of_head<ROWS>(request_of(p, i), p.G) * p.H_kv : 0; };
  auto take_share = [&](long long total) {
    const long long share = share_of(total, p.workgroups);
    at = share * blockIdx.x;
    end = min(at + share, total);
    if (blockIdx.x == 0 && threadIdx.x == 0) p.first_unit[p.R] = total;
  };
  if (p.R <= kWave) {  // every wave for itself, nothing through LDS
    const long long w = work_of(lane), until = wave_scan(w);
    if (blockIdx.x == 0 && wave == 0 && lane < p.R) p.first_unit[lane] = until - w;
    take_share(read_lane64(until, kWave - 1));
    if (at >= end) return;
    r = __builtin_ctzll(__ballot(at < until));
    rest = at - read_lane64(until - w, r);
  } else {
    long long total = 0;
    for (int base = 0; base < p.R; base += kThreads) {
      const int i = base + threadIdx.x;
      const long long w = work_of(i), before = total + block_scan(w, lane, wave, scan, &total);
      if (blockIdx.x == 0 && i < p.R) p.first_unit[i] = before;
    }
    take_share(total);
    if (at >= end) return;
    long long carry = 0;
    for (int base = 0; base < p.R && at >= carry; base += kThreads) {
      const long long w = work_of(base + threadIdx.x), before = carry + block_scan(w, lane, wave, scan, &carry);
      if (at >= before && at < before + w) {
        found[0] = base + threadIdx.x;
        found[1] = at - before;
      }
    }
    __syncthreads();
    r = __builtin_amdgcn_readfirstlane(static_cast<int>(found[0]));
    rest = read_lane64(found[1], 0);
  }
  Request rq = request_of(p, r);
  int tiles = tiles_of<ROWS>(rq, p.G);
  const long long per_head = units_of_head<ROWS>(rq, p.G);
  int head = static_cast<int>(quotient(rest, per_head));
  rest -= head * per_head;
  int tile = 0;
  for (;; ++tile) {
    const int n = blocks_of<ROWS>(rq, p.G, tile) + kItemUnits;
    if (rest < n) break;
    rest -= n;
  }

  while (true) {
    const int n_blocks = blocks_of<ROWS>(rq, p.G, tile);
    const int b0 = max(static_cast<int>(rest) - kItemUnits, 0);
    const int b1 = static_cast<int>(min(rest + (end - at) - kItemUnits, static_cast<long long>(n_blocks)));
    if (b1 <= b0) return;  // only units that stand for no block are left
    const int rows = min(rq.q_len * p.G - tile * ROWS, ROWS);

    // ---- queries: B operands, columns are query rows
    bf16x8 q[NC][kTerms][kSteps];
    int last_key[NC];  // last key that the column's row sees
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      const int in_tile = s * COLS + (PAIRED ? c & 7 : c);
      const int row = tile * ROWS + in_tile;
      const bool exists = in_tile < rows;
      const int token = row / p.G, h = row - token * p.G;
      last_key[s] = exists ? rq.len - rq.q_len + token : -1;
      const char* src = p.q.token(rq.first_row + (exists ? token : 0)) + (head * p.G + (exists ? h : 0)) * p.q.head_stride;
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        const int ch = D == 128 ? 32 * kg + 8 * j : 16 * kg + 8 * j;
        if constexpr (sizeof(T) == 2) {
          q[s][0][j] = *reinterpret_cast<const bf16x8*>(src + ch * 2);
        } else {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = reinterpret_cast<const float*>(src)[ch + i];
#pragma unroll
          for (int t = 0; t < 3; ++t) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
              x[2 * i] -= low_half(w[i]);
              x[2 * i + 1] -= high_half(w[i]);
            }
            q[s][t][j] = words_to_bf16x8(w[0], w[1], w[2], w[3]);
          }
        }
      }
    }
    // Blocks whose keys every row sees need no mask.
    const int open = visible(rq, tile * ROWS / p.G) / kKv4Block;

    floatx4 o[NC][kFrags], l[NC];  // l: sums of weights, by a product with ones; all four the same
    float m[NC];
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      m[s] = kLowest;
      l[s] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int f = 0; f < kFrags; ++f) o[s][f] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    const int32_t* table = p.block_table + static_cast<size_t>(r) * p.max_pages;
    const int page_shift = p.cache.page_shift - 5;
    int pages = 0;       // lane i: page of this wave's block number first + i
    int first = 0;
    auto page_of = [&](int i) {  // of the wave's block number i
      if ((i & 63) == 0) {
        first = i;
        pages = table[min((b0 + wave + (first + lane) * kWaves) >> page_shift, p.max_pages - 1)];
      }
      return __builtin_amdgcn_readlane(pages, i & 63);
    };
    uint32_t nowhere = 0;  // bit i: the table names no page for the block in slot i of the ring
    auto request = [&](int i) {
      const int blk = b0 + wave + i * kWaves, slot = i % R::kDepth;
      const int page = page_of(i);
      const bool exists = page >= 0 && page < p.cache.n_pages;
      nowhere = (nowhere & ~(1u << slot)) | (exists ? 0u : 1u << slot);
      request_block<D>(p.cache.base + kv4_block_offset<D>(p.cache, exists ? page : 0, head, blk & ((1 << page_shift) - 1)),
                       ring + slot * R::kSlot, key_piece, straight, word);
    };
    const int mine = (b1 - b0 - wave + kWaves - 1) / kWaves;  // blocks of this wave (may be none)
    for (int i = 0; i < min(mine, R::kDepth); ++i) request(i);
    for (int i = 0; i < mine; ++i) {
      const int blk = b0 + wave + i * kWaves;
      const int key0 = blk * kKv4Block;
      const int slot = i % R::kDepth;
      const bool ok = !(nowhere >> slot & 1u), masked = !ok || blk >= open;
      wait_block<D>(min(mine - 1 - i, R::kDepth - 1));
      BlockData<D> b;
      read_block<D>(ring + slot * R::kSlot, lane, b);
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the slot is free again
      if (i + R::kDepth < mine) request(i + R::kDepth);

      // S^T: rows are tokens a * 16 + 4 kg + i
      floatx4 z[NC][2];
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const float scale = kv4_scale(b.ks[a]);
#pragma unroll
        for (int s = 0; s < NC; ++s) z[s][a] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          const bf16x8 row = decode_word(b.k[a][j], scale);
#pragma unroll
          for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int t = 0; t < kTerms; ++t) z[s][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(row, q[s][t][j], z[s][a], 0, 0, 0);
        }
      }
      bool not_finite = false;  // values that are not and that some row must not see
      if (masked) {
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
          for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!ok || key0 + a * 16 + 4 * kg + e > last_key[s]) z[s][a][e] = -INFINITY;
        // what lies past the request's tokens may be anything
        uint32_t any = 0;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!ok || key0 + a * 16 + 4 * kg + e >= rq.len) {
              b.v[a][e] = 0u;
              b.vs[a] = (b.vs[a] & ~(0xffu << (8 * e))) | (127u << (8 * e));
            }
          // a byte of 255 is the only one that grows past its top bit here
          any |= (((b.vs[a] & 0x7f7f7f7fu) + 0x01010101u) & b.vs[a]) & 0x80808080u;
        }
        not_finite = __any(any != 0);
      }

      // weights
      bf16x8 w[NC][kParts];
#pragma unroll
      for (int s = 0; s < NC; ++s) {
        // (of a NaN and a number the NaN, in one instruction for three: a row with one is NaN whatever its reference)
        float top = z[s][0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = __builtin_elementwise_maximum(top, z[s][e / 4][e % 4]);
        top *= p.scale_log2;
        if (__any(top > m[s] + kSlack)) {
          const float grown = fmaxf(m[s], max_across_rows(top)), shrink = __builtin_amdgcn_exp2f(m[s] - grown);
          m[s] = grown;
          l[s] *= shrink;
#pragma unroll
          for (int f = 0; f < kFrags; ++f) o[s][f] *= shrink;
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(z[s][e / 4][e % 4], p.scale_log2, -m[s]));
        // number t of a weight: what is left of it after those before, rounded
        uint32_t part[3][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int t = 0; t < kNumbers; ++t) {
            part[t][e] = pack_bf16(x[2 * e], x[2 * e + 1]);
            if (t + 1 == kNumbers) break;
            if (PAIRED && t == 0) {  // taken off in the upper columns only: in the lower ones the next number is the first
              x[2 * e] = less(x[2 * e], part[t][e], upper_low);
              x[2 * e + 1] = less(x[2 * e + 1], part[t][e], upper_high);
            } else {
              x[2 * e] = less(x[2 * e], part[t][e], low);
              x[2 * e + 1] = less(x[2 * e + 1], part[t][e], high);
            }
          }
          if constexpr (PAIRED && kNumbers == 3) {
            // lower: part[1] is the first, part[2] the second of it; upper: part[1] the second, part[2] the third
            part[0][e] = part[1][e];
            part[1][e] = c < 8 ? 0u : part[2][e];
          } else if constexpr (PAIRED) {
            part[0][e] = part[1][e];
          }
        }
#pragma unroll
        for (int t = 0; t < kParts; ++t) {
          w[s][t] = words_to_bf16x8(part[t][0], part[t][1], part[t][2], part[t][3]);
          l[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, w[s][t], l[s], 0, 0, 0);
        }
      }

      // O^T
      float scale[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)  // (the conversion looks at the exponent alone: what is beside the byte does not matter)
        scale[e] = __uint_as_float(e % 4 == 3 ? b.vs[e / 4] >> 1 : b.vs[e / 4] << (23 - 8 * (e % 4)));
      if (not_finite) {
        // A NaN in a product of zero weight would reach the rows that do not see its token: it is taken out of the values,
        // and an output that has weight on it becomes NaN below.
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (((b.vs[e / 4] >> (8 * (e % 4))) & 0xffu) == kKv4NotFinite) {
            b.v[e / 4][e % 4] = 0u;
            scale[e] = 1.f;
          }
      }
      auto accumulate = [&](auto pair_constant) {  // channels 2 * pair and 2 * pair + 1 of every chunk
        constexpr int pair = decltype(pair_constant)::value;
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b.v[e / 4][e % 4], scale[e], pair));
        // D = 128: both channels in turn.  D = 64: lanes 0..7 the even one of their chunk, lanes 8..15 the odd one.
#pragma unroll
        for (int half = 0; half < (D == 128 ? 2 : 1); ++half) {
          const int f = D == 128 ? 2 * pair + half : pair;
          const uint32_t take = (D == 128 ? half != 0 : c >= 8) ? 0x07060302u : 0x05040100u;
          const bf16x8 a = words_to_bf16x8(__builtin_amdgcn_perm(v[1], v[0], take), __builtin_amdgcn_perm(v[3], v[2], take),
                                           __builtin_amdgcn_perm(v[5], v[4], take), __builtin_amdgcn_perm(v[7], v[6], take));
#pragma unroll
          for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int t = 0; t < kParts; ++t) o[s][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[s][t], o[s][f], 0, 0, 0);
        }
      };
      accumulate(Constant<0>{});
      accumulate(Constant<1>{});
      accumulate(Constant<2>{});
      accumulate(Constant<3>{});
      if (not_finite) {
        uint32_t ones[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const uint32_t pair = b.vs[e / 4] >> (8 * (e % 4));
          ones[e / 2] = ((pair & 0xffu) == kKv4NotFinite ? 0x3f80u : 0u) | ((pair >> 8 & 0xffu) == kKv4NotFinite ? 0x3f800000u : 0u);
        }
        const bf16x8 n = words_to_bf16x8(ones[0], ones[1], ones[2], ones[3]);
#pragma unroll
        for (int s = 0; s < NC; ++s) {  // weight on such tokens, of a chunk's channels
          const floatx4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(n, w[s][0], (floatx4{0.f, 0.f, 0.f, 0.f}), 0, 0, 0);
#pragma unroll
          for (int f = 0; f < kFrags; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[s][f][e] = hit[e] != 0.f ? NAN : o[s][f][e];
        }
      }
    }

    // ---- join the waves: every wave has read all of its ring
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      if (lane < COLS) sh_m[wave][s * COLS + c] = m[s];
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      const int row = s * COLS + (PAIRED ? c & 7 : c);
      float all = sh_m[0][row];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) all = fmaxf(all, sh_m[i][row]);
      const float shrink = __builtin_amdgcn_exp2f(m[s] - all);
      m[s] = all;
      float weights = l[s][0] * shrink;
      if constexpr (PAIRED) weights += __uint_as_float(lane_xor<8>(__float_as_uint(weights)));
      if (lane < COLS) sh_l[wave][row] = weights;
#pragma unroll
      for (int f = 0; f < kFrags; ++f)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = o[s][f][e] * shrink;
          if constexpr (PAIRED) x += __uint_as_float(lane_xor<8>(__float_as_uint(x)));
          const int a_row = 4 * kg + e;
          const int ch = D == 128 ? 8 * a_row + f : (a_row & 7) * 8 + 2 * f + (a_row >> 3);
          if (!PAIRED || c < 8) sh_o[wave][row][ch] = x;
        }
    }
    __syncthreads();
    const bool whole = b0 == 0 && b1 == n_blocks;
    const size_t part = 2 * static_cast<size_t>(blockIdx.x) + (b0 == 0 ? 1 : 0);
    for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
      const int row = i / (D / 4), ch = i % (D / 4) * 4;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f, top = sh_m[0][row];
#pragma unroll
      for (int j = 0; j < kWaves; ++j) {
        const float4 y = *reinterpret_cast<const float4*>(&sh_o[j][row][ch]);
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
        sum += sh_l[j][row];
        top = fmaxf(top, sh_m[j][row]);
      }
      if (whole) {
        write_row<T>(p, rq, head, tile * ROWS + row, ch, x, top, sum);
      } else {
        *reinterpret_cast<float4*>(p.part_o + (part * ROWS + row) * D + ch) = x;
        if (ch == 0) p.part_ml[part * ROWS + row] = make_float2(top, sum);
      }
    }
    at += n_blocks + kItemUnits - rest;
    if (at >= end) return;
    __syncthreads();
    // the next item
    rest = 0;
    if (++tile == tiles) {
      tile = 0;
      if (++head == p.H_kv) {
        head = 0;
        do {
          rq = request_of(p, ++r);
          tiles = tiles_of<ROWS>(rq, p.G);
        } while (tiles == 0);
      }
    }
  }
}

// Joins the parts of the items that several workgroups shared: workgroup (request * H_kv + head, tile).  The threads of a
// row's four channels share its parts, four of them in flight each, every thread with a maximum of its own.
constexpr int kJoinThreads = 1024;
template <int D, typename T, int ROWS>
__global__ __launch_bounds__(kJoinThreads) void kv4_join_kernel(Params p) {
  constexpr int kCells = ROWS * (D / 4), kShares = kJoinThreads / kCells;
  static_assert(kShares >= 1, "a thread has four channels of one row");
  __shared__ __align__(16) float4 sh_x[kJoinThreads];
  __shared__ float2 sh_ml[kJoinThreads];
  const int r = blockIdx.x / p.H_kv, head = blockIdx.x % p.H_kv, tile = blockIdx.y;
  const Request rq = request_of(p, r);
  if (tile >= tiles_of<ROWS>(rq, p.G)) return;
  const long long total = p.first_unit[p.R];
  const long long share = share_of(total, p.workgroups);
  long long at = p.first_unit[r];
  if (head) at += head * units_of_head<ROWS>(rq, p.G);
  for (int t = 0; t < tile; ++t) at += blocks_of<ROWS>(rq, p.G, t) + kItemUnits;
  at += kItemUnits;  // its first block
  const long long last = at + blocks_of<ROWS>(rq, p.G, tile) - 1;
  const int w0 = static_cast<int>(quotient(at, share)), w1 = static_cast<int>(quotient(last, share));
  if (w0 == w1) return;  // one workgroup had all of it
  const int rows = min(rq.q_len * p.G - tile * ROWS, ROWS);
  const int cell = threadIdx.x % kCells, row = cell / (D / 4), ch = cell % (D / 4) * 4;
  float top = kLowest, sum = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  if (row < rows) {
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
  if (row >= rows) return;
  write_row<T>(p, rq, head, tile * ROWS + row, ch, x, top, sum);
}

// Rows of a tile: as many as a request has, up to 32.
int rows_of_tile(const Kv4AttentionArgs& a) {
  const long long rows = static_cast<long long>(a.max_q_len) * a.G;
  return rows <= 8 ? 8 : rows <= 16 ? 16 : 32;
}

// Workgroups of a launch: those that run at once (a second round would have its first trips to memory by itself), and no
// more than can have kMinUnits each.
int workgroups_of(const Kv4AttentionArgs& a, int rows) {
  const long long tiles = (static_cast<long long>(a.max_q_len) * a.G + rows - 1) / rows;
  const long long longest = (static_cast<long long>(a.max_pages) << a.cache.page_shift) / kKv4Block;
  const double units = static_cast<double>(a.R) * a.H_kv * tiles * (longest + kItemUnits);
  return static_cast<int>(fmin(fmax(ceil(units / kMinUnits), 1.0), static_cast<double>(kCus * workgroups_per_cu(a.dtype == SHOTKV_F32, rows))));
}

struct Workspace {
  long long* first_unit;
  float2* part_ml;
  float* part_o;
  size_t bytes;
};
Workspace carve(const Kv4AttentionArgs& a, void* base) {
  const int rows = rows_of_tile(a), workgroups = workgroups_of(a, rows);
  Workspace w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* ptr = base ? static_cast<char*>(base) + off : nullptr;
    off = align_up(off + bytes, 256);
    return ptr;
  };
  w.first_unit = reinterpret_cast<long long*>(take((static_cast<size_t>(a.R) + 1) * 8));
  w.part_ml = reinterpret_cast<float2*>(take(static_cast<size_t>(2) * workgroups * rows * 8));
  w.part_o = reinterpret_cast<float*>(take(static_cast<size_t>(2) * workgroups * rows * a.D * 4));
  w.bytes = off;
  return w;
}

template <int D, typename T, int NC, bool PAIRED>
hipError_t launch(const Params& p, hipStream_t s) {
  constexpr int rows = (PAIRED ? 8 : 16) * NC;
  kv4_attention_kernel<D, T, NC, PAIRED><<<p.workgroups, kThreads, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.workgroups == 1) return e;
  const int tiles = ceil_div(p.max_q_len * p.G, rows);
  kv4_join_kernel<D, T, rows><<<dim3(p.R * p.H_kv, tiles), kJoinThreads, 0, s>>>(p);
  return hipGetLastError();
}

template <int D>
hipError_t launch_rows(const Kv4AttentionArgs& a, const Params& p, hipStream_t s) {
  const int rows = rows_of_tile(a);
  if (a.dtype == SHOTKV_F32) {
    if (rows == 8) return launch<D, float, 1, true>(p, s);
    return rows == 16 ? launch<D, float, 1, false>(p, s) : launch<D, float, 2, false>(p, s);
  }
  if (rows == 8) return launch<D, bf16_t, 1, true>(p, s);
  return rows == 16 ? launch<D, bf16_t, 1, false>(p, s) : launch<D, bf16_t, 2, false>(p, s);
}

}  // namespace

size_t kv4_attention_workspace(const Kv4AttentionArgs& a) { return carve(a, nullptr).bytes; }

hipError_t launch_kv4_attention(const Kv4AttentionArgs& a, void* workspace, hipStream_t s) {
  const Workspace w = carve(a, workspace);
  Params p{};
  p.R = a.R; p.T = a.T; p.H = a.H; p.H_kv = a.H_kv; p.G = a.G; p.max_q_len = a.max_q_len; p.max_pages = a.max_pages;
  p.workgroups = workgroups_of(a, rows_of_tile(a));
  p.scale_log2 = a.sm_scale * kLog2e;
  p.cache = a.cache;
  p.block_table = a.block_table; p.seq_lens = a.seq_lens; p.query_start = a.query_start;
  p.q = a.q; p.out = a.out; p.lse = a.lse;
  p.first_unit = w.first_unit; p.part_ml = w.part_ml; p.part_o = w.part_o;
  return a.D == 128 ? launch_rows<128>(a, p, s) : launch_rows<64>(a, p, s);
}

}  // namespace shotkv
