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
// would be off by up to 2^-8, as much as the output's own rounding): what the first leaves goes through the second product
// once more.  Up to eight rows leave half of the columns empty; there columns 8..15 repeat the query rows of columns 0..7
// and hold the second numbers (PAIRED), at no further matrix work.  fp32 queries are the sum of three bf16 numbers, in three
// products.
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
constexpr int kMaxWorkgroups = 1024;  // four to a CU
constexpr int kMinBlocks = 8;         // of a workgroup: two to a wave
constexpr float kLowest = -1e30f;     // a running maximum before any key
constexpr float kLn2 = 0.6931471805599453f;

struct Params {
  int R, T, H, H_kv, G, max_q_len, max_pages, workgroups;
  float scale_log2;
  Kv4Pages cache;
  const int32_t *block_table, *seq_lens, *query_start;
  RowView q, out;
  float* lse;
  long long* first_block;  // [R + 1] blocks before each request
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
template <int ROWS>
__device__ __forceinline__ long long blocks_of_head(const Request& q, int G) {
  const int tiles = tiles_of<ROWS>(q, G);
  long long sum = 0;
  for (int t = 0; t < tiles; ++t) sum += blocks_of<ROWS>(q, G, t);
  return sum;
}

__device__ __forceinline__ long long shfl_up64(long long v, int d) { return __shfl_up(v, d); }

// Loads of one block by one wave.
template <int D>
struct BlockLoad {
  uint32_t k[2][D / 32];   // two times 16 tokens: this lane's codes of its token
  uint32_t ks[2];
  u32x4 v[2];              // two quads of tokens: this lane's chunk of channels
  uint32_t vs[2];
};

template <int D>
__device__ __forceinline__ void load_block(const char* __restrict__ base, int lane, BlockLoad<D>& b) {
  typedef Kv4Block<D> B;
  const int c = lane & 15, kg = lane >> 4;
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    const int token = a * 16 + c;
    if constexpr (D == 128) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(base + B::kKeys + token * 64 + kg * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) b.k[a][j] = w[j];
      b.ks[a] = *reinterpret_cast<const uint8_t*>(base + B::kKeyScales + token * 4 + kg);
    } else {
      const u32x2 w = *reinterpret_cast<const u32x2*>(base + B::kKeys + token * 32 + kg * 8);
      b.k[a][0] = w[0];
      b.k[a][1] = w[1];
      b.ks[a] = *reinterpret_cast<const uint8_t*>(base + B::kKeyScales + token * 2 + kg / 2);
    }
    const int quad = a * 4 + kg, chunk = c % (D / 8);
    b.v[a] = *reinterpret_cast<const u32x4*>(base + B::kValues + (quad * (D / 8) + chunk) * 16);
    b.vs[a] = *reinterpret_cast<const uint32_t*>(base + B::kValueScales + (quad * (D / 32) + chunk / 4) * 4);
  }
}

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
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ float max_across_rows(float x) {  // over lanes 16, 32 and 48 away
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_across_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_across_rows(float x) { return sum_across_halves(sum_across_row_pairs(x)); }

// T: storage type of queries and output.  COLS: query rows of a set of 16 columns (8 if PAIRED).  NC: sets of columns.
template <int D, typename T, int NC, bool PAIRED>
__global__ __launch_bounds__(kThreads) void kv4_attention_kernel(Params p) {
  constexpr int COLS = PAIRED ? 8 : 16, ROWS = COLS * NC;
  constexpr int kSteps = D / 32;                    // of the first product
  constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;    // bf16 numbers that a query element is the sum of
  constexpr int kParts = PAIRED ? 1 : 2;            // products that a weight goes through
  constexpr int kFrags = D / 16;                    // 16 channels each of the second product
  constexpr int kPad = D + 4;
  __shared__ long long scan[kWaves + 1];
  __shared__ long long found[2];
  __shared__ float sh_m[kWaves][ROWS], sh_l[kWaves][ROWS];
  __shared__ __align__(16) float sh_o[kWaves][ROWS][kPad];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = lane & 15, kg = lane >> 4;

  // ---- this workgroup's share of the blocks
  long long total = 0;
  for (int base = 0; base < p.R; base += kThreads) {
    const int r = base + threadIdx.x;
    long long w = r < p.R ? blocks_of_head<ROWS>(request_of(p, r), p.G) * p.H_kv : 0, sum = w;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const long long up = shfl_up64(sum, d);
      if (lane >= d) sum += up;
    }
    __syncthreads();
    if (lane == kWave - 1) scan[wave] = sum;
    __syncthreads();
    long long before = total;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      if (i < wave) before += scan[i];
      total += scan[i];
    }
    if (r < p.R && blockIdx.x == 0) p.first_block[r] = before + sum - w;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.first_block[p.R] = total;
  const long long share = max((total + p.workgroups - 1) / p.workgroups, static_cast<long long>(kMinBlocks));
  long long at = share * blockIdx.x;
  const long long end = min(at + share, total);
  if (at >= end) return;
  // the request that holds block `at`, and what of it lies before
  long long carry = 0;
  for (int base = 0; base < p.R; base += kThreads) {
    const int r = base + threadIdx.x;
    long long w = r < p.R ? blocks_of_head<ROWS>(request_of(p, r), p.G) * p.H_kv : 0, sum = w;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const long long up = shfl_up64(sum, d);
      if (lane >= d) sum += up;
    }
    __syncthreads();
    if (lane == kWave - 1) scan[wave] = sum;
    __syncthreads();
    long long before = carry;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      if (i < wave) before += scan[i];
      carry += scan[i];
    }
    before += sum - w;
    if (at >= before && at < before + w) {
      found[0] = r;
      found[1] = at - before;
    }
    if (at < carry) break;
  }
  __syncthreads();
  int r = __builtin_amdgcn_readfirstlane(static_cast<int>(found[0]));
  long long rest = found[1];
  Request rq = request_of(p, r);
  int tiles = tiles_of<ROWS>(rq, p.G);
  const long long per_head = blocks_of_head<ROWS>(rq, p.G);
  int head = static_cast<int>(rest / per_head);
  rest -= head * per_head;
  int tile = 0, b0 = 0;
  for (;; ++tile) {
    const int n = blocks_of<ROWS>(rq, p.G, tile);
    if (rest < n) break;
    rest -= n;
  }
  b0 = static_cast<int>(rest);

  while (true) {
    const int n_blocks = blocks_of<ROWS>(rq, p.G, tile);
    const int b1 = static_cast<int>(min(static_cast<long long>(n_blocks), b0 + (end - at)));
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

    floatx4 o[NC][kFrags];
    float m[NC], l[NC];
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      m[s] = kLowest;
      l[s] = 0.f;
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
    auto fetch = [&](int i, BlockLoad<D>& b) {  // whether the page exists
      const int blk = b0 + wave + i * kWaves;
      const int page = page_of(i);
      const bool ok = page >= 0 && page < p.cache.n_pages;
      load_block<D>(p.cache.base + kv4_block_offset<D>(p.cache, ok ? page : 0, head, blk & ((1 << page_shift) - 1)), lane, b);
      return ok;
    };
    const int mine = (b1 - b0 - wave + kWaves - 1) / kWaves;  // blocks of this wave (may be none)
    BlockLoad<D> next;
    bool next_ok = false;
    if (mine > 0) next_ok = fetch(0, next);
    for (int i = 0; i < mine; ++i) {
      BlockLoad<D> b = next;
      const bool ok = next_ok;
      if (i + 1 < mine) next_ok = fetch(i + 1, next);
      const int blk = b0 + wave + i * kWaves;
      const int key0 = blk * kKv4Block;
      const bool masked = !ok || blk >= open;

      // S^T: rows are tokens a * 16 + 4 kg + i
      floatx4 z[NC][2];
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const float scale = kv4_scale(b.ks[a]);
#pragma unroll
        for (int s = 0; s < NC; ++s) z[s][a] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          const bf16x8 k = decode_word(b.k[a][j], scale);
#pragma unroll
          for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int t = 0; t < kTerms; ++t) z[s][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[s][t][j], z[s][a], 0, 0, 0);
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
        float top = fmaxf(fmaxf(fmaxf(z[s][0][0], z[s][0][1]), fmaxf(z[s][0][2], z[s][0][3])),
                          fmaxf(fmaxf(z[s][1][0], z[s][1][1]), fmaxf(z[s][1][2], z[s][1][3])));
        top = max_across_rows(top) * p.scale_log2;
        if (__any(top > m[s])) {
          const float grown = fmaxf(m[s], top), shrink = __builtin_amdgcn_exp2f(m[s] - grown);
          m[s] = grown;
          l[s] *= shrink;
#pragma unroll
          for (int f = 0; f < kFrags; ++f) o[s][f] *= shrink;
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = __builtin_amdgcn_exp2f(fmaf(z[s][e / 4][e % 4], p.scale_log2, -m[s]));
          l[s] += x[e];
        }
        uint32_t words[4], left[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          words[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
          const uint32_t taken = !PAIRED || c >= 8 ? words[e] : 0u;
          left[e] = pack_bf16(x[2 * e] - low_half(taken), x[2 * e + 1] - high_half(taken));
        }
        if constexpr (PAIRED) {
          w[s][0] = words_to_bf16x8(left[0], left[1], left[2], left[3]);  // (of the lower columns all is left)
        } else {
          w[s][0] = words_to_bf16x8(words[0], words[1], words[2], words[3]);
          w[s][1] = words_to_bf16x8(left[0], left[1], left[2], left[3]);
        }
      }

      // O^T
      uint32_t v[8][4];  // [token][pairs of channels]
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float scale = kv4_scale((b.vs[e / 4] >> (8 * (e % 4))) & 0xffu);
        const uint32_t codes = b.v[e / 4][e % 4];
        v[e][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
        v[e][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
        v[e][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
        v[e][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
      }
      uint32_t bad[8];
      if (not_finite) {
        // A NaN in a product of zero weight would reach the rows that do not see its token: it is taken out of the values,
        // and an output that has weight on it becomes NaN below.
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          bad[e] = ((b.vs[e / 4] >> (8 * (e % 4))) & 0xffu) == kKv4NotFinite ? 0x3f803f80u : 0u;
          if (bad[e])
#pragma unroll
            for (int j = 0; j < 4; ++j) v[e][j] = 0u;
        }
      }
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        // D = 128: channel 8 c + f.  D = 64: lanes 0..7 the even channel of pair f of their chunk, lanes 8..15 the odd one.
        const int pair = D == 128 ? f / 2 : f;
        const uint32_t take = (D == 128 ? f % 2 : c >= 8) ? 0x07060302u : 0x05040100u;
        const bf16x8 a = words_to_bf16x8(
            __builtin_amdgcn_perm(v[1][pair], v[0][pair], take), __builtin_amdgcn_perm(v[3][pair], v[2][pair], take),
            __builtin_amdgcn_perm(v[5][pair], v[4][pair], take), __builtin_amdgcn_perm(v[7][pair], v[6][pair], take));
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
          for (int t = 0; t < kParts; ++t) o[s][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[s][t], o[s][f], 0, 0, 0);
        if (not_finite) {
          const bf16x8 n = words_to_bf16x8(__builtin_amdgcn_perm(bad[1], bad[0], take), __builtin_amdgcn_perm(bad[3], bad[2], take),
                                           __builtin_amdgcn_perm(bad[5], bad[4], take), __builtin_amdgcn_perm(bad[7], bad[6], take));
#pragma unroll
          for (int s = 0; s < NC; ++s) {
            const floatx4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(n, w[s][0], (floatx4{0.f, 0.f, 0.f, 0.f}), 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[s][f][e] = hit[e] != 0.f ? NAN : o[s][f][e];
          }
        }
      }
    }

    // ---- join the waves
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      l[s] = sum_across_rows(l[s]);
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
      if (lane < COLS) sh_l[wave][row] = l[s] * shrink;
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
        const int flat = tile * ROWS + row, token = flat / p.G, h = flat - token * p.G;
        const float inv = sum != 0.f ? 1.f / sum : 0.f;
        char* dst = p.out.token(rq.first_row + token) + (head * p.G + h) * p.out.head_stride;
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<u32x2*>(dst + ch * 2) = u32x2{pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv)};
        } else {
          *reinterpret_cast<float4*>(dst + ch * 4) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
        }
        if (ch == 0 && p.lse)
          p.lse[static_cast<size_t>(rq.first_row + token) * p.H + head * p.G + h] = sum != 0.f ? add_log2(top, sum) * kLn2 : -INFINITY;
      } else {
        *reinterpret_cast<float4*>(p.part_o + (part * ROWS + row) * D + ch) = x;
        if (ch == 0) p.part_ml[part * ROWS + row] = make_float2(top, sum);
      }
    }
    at += b1 - b0;
    if (at >= end) return;
    __syncthreads();
    // the next item
    b0 = 0;
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

// Joins the parts of the items that several workgroups shared: workgroup (request * H_kv + head, tile).
template <int D, typename T, int ROWS>
__global__ __launch_bounds__(kThreads) void kv4_join_kernel(Params p) {
  const int r = blockIdx.x / p.H_kv, head = blockIdx.x % p.H_kv, tile = blockIdx.y;
  const Request rq = request_of(p, r);
  if (tile >= tiles_of<ROWS>(rq, p.G)) return;
  const long long total = p.first_block[p.R];
  const long long share = max((total + p.workgroups - 1) / p.workgroups, static_cast<long long>(kMinBlocks));
  long long at = p.first_block[r] + head * blocks_of_head<ROWS>(rq, p.G);
  for (int t = 0; t < tile; ++t) at += blocks_of<ROWS>(rq, p.G, t);
  const long long last = at + blocks_of<ROWS>(rq, p.G, tile) - 1;
  const int w0 = static_cast<int>(at / share), w1 = static_cast<int>(last / share);
  if (w0 == w1) return;  // one workgroup had all of it
  const int rows = min(rq.q_len * p.G - tile * ROWS, ROWS);
  for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
    const int row = i / (D / 4), ch = i % (D / 4) * 4;
    // the first part is the one that begins the item, the others are their workgroups' first
    auto part_of = [&](int w) { return 2 * static_cast<size_t>(w) + (w == w0 ? 1 : 0); };
    float top = kLowest;
    for (int w = w0; w <= w1; ++w) top = fmaxf(top, p.part_ml[part_of(w) * ROWS + row].x);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
    for (int w = w0; w <= w1; ++w) {
      const float2 ml = p.part_ml[part_of(w) * ROWS + row];
      const float4 y = *reinterpret_cast<const float4*>(p.part_o + (part_of(w) * ROWS + row) * D + ch);
      const float f = __builtin_amdgcn_exp2f(ml.x - top);
      x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
      sum = fmaf(ml.y, f, sum);
    }
    const int flat = tile * ROWS + row, token = flat / p.G, h = flat - token * p.G;
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
}

// Rows of a tile: as many as a request has, up to 32.
int rows_of_tile(const Kv4AttentionArgs& a) {
  const long long rows = static_cast<long long>(a.max_q_len) * a.G;
  return rows <= 8 ? 8 : rows <= 16 ? 16 : 32;
}

// Workgroups of a launch: no more than can have kMinBlocks each.
int workgroups_of(const Kv4AttentionArgs& a, int rows) {
  const long long tiles = (static_cast<long long>(a.max_q_len) * a.G + rows - 1) / rows;
  const long long longest = (static_cast<long long>(a.max_pages) << a.cache.page_shift) / kKv4Block;
  const double blocks = static_cast<double>(a.R) * a.H_kv * tiles * longest;
  return static_cast<int>(fmin(fmax(ceil(blocks / kMinBlocks), 1.0), static_cast<double>(kMaxWorkgroups)));
}

struct Workspace {
  long long* first_block;
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
  w.first_block = reinterpret_cast<long long*>(take((static_cast<size_t>(a.R) + 1) * 8));
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
  kv4_join_kernel<D, T, rows><<<dim3(p.R * p.H_kv, tiles), kThreads, 0, s>>>(p);
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
  p.first_block = w.first_block; p.part_ml = w.part_ml; p.part_o = w.part_o;
  return a.D == 128 ? launch_rows<128>(a, p, s) : launch_rows<64>(a, p, s);
}

}  // namespace shotkv
