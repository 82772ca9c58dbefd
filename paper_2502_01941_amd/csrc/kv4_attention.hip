// Attention of up to 32 query rows per KV head over the paged 4-bit cache: single tokens and drafts.
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
// The four waves of a workgroup take blocks in turn, each through a ring of its own in LDS, and join their sums at the end.
//
// Bound by the stream of blocks where it is long, by dependent trips to memory (lengths, page, block, parts) where it is short.
// bf16, 32 heads over 8, 128 channels, kernel and join: 64 requests of 200 to 32768 tokens (437 MB) 76 + 4.5 us, 5.7 TB/s, what
// the same loads without the arithmetic take; 16 of 4096 to 5120 (80 MB) 20 + 4.5; one of 3277 (3.6 MB) 7 + 3, of which a launch
// and the first block are 5.
//
// Precision: sums, maxima and the output are 32-bit.  A weight is the sum of two bf16 numbers (2^-16 off at most; as one it
// would be off by up to 2^-8, as much as a bf16 output's own rounding), of three where the output is fp32: what the first
// leaves goes through the second product once more.  Their sums are of the numbers that the values are weighted with (the kernel
// for many rows adds them before they are rounded); a bf16 call's lse has up to 2^-17 from that.  Up to eight rows leave half of the columns empty; there columns 8..15
// repeat the query rows of columns 0..7 and hold the second numbers (PAIRED), at no further matrix work.  fp32 queries are
// the sum of three bf16 numbers, in three products.
#include "kv4_attention.hpp"

namespace shotkv {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
// Two blocks to a wave: 16 requests of 4096 with 8 new tokens take 32.6 us, with three 35.6 (more LDS for each workgroup's
// start), and a fourth costs a workgroup of the CU: 64 single tokens of 200 to 32768 86, 88 and 120 us.
constexpr int kRingBlocks = 2;
// An item's start and end count for 16 blocks (16 requests of about 4600 tokens take 25.5 us with 8 as well), and a workgroup has
// at least half as many units (one request of 3277 tokens: 4 10.9 us, 8 10.2, 16 11.6).
constexpr int kItemUnits = 16, kMinUnits = 8;

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
// The oldest block has arrived; `more`: there is a younger one.
template <int D>
__device__ __forceinline__ void wait_block(bool more) {
  static_assert(kRingBlocks == 2, "one block besides the oldest");
  if (more) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(Ring<D>::kLoads) : "memory");
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

__device__ __forceinline__ bf16x8 decode_word(uint32_t codes, float scale) {
  return words_to_bf16x8(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)));
}
__device__ __forceinline__ float max_across_rows(float x) {  // over lanes 16, 32 and 48 away
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_across_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// Workgroups of a CU at once: four waves each, of up to 168 registers in the forms for up to 16 rows in bf16 (of 128, four at
// once, they spill: 100 us for 89), of up to 256 in the others (the one for 32 rows of 128 channels in fp32 spills 22).
constexpr int workgroups_per_cu(bool f32, int rows) { return f32 || rows > 16 ? 2 : 3; }

// T: storage type of queries and output.  COLS: query rows of a set of 16 columns (8 if PAIRED).  NC: sets of columns.
template <int D, typename T, int NC, bool PAIRED>
__global__ __launch_bounds__(kThreads, workgroups_per_cu(sizeof(T) == 4, (PAIRED ? 8 : 16) * NC)) void kv4_attention_kernel(AttnParams p) {
  constexpr int COLS = PAIRED ? 8 : 16, ROWS = COLS * NC;
  typedef Division<ROWS, kItemUnits, kMinUnits> Div;
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
  long long at, end, rest, share, per_head;
  int r;
  Request rq;
  if (threadIdx.x == 0) p.cut[blockIdx.x].rows = 0;
  auto blocks_of = [](const Request& q) { return max((q.len + kKv4Block - 1) / kKv4Block, 1); };  // its last row sees all of it
  auto units_of_head = [&](const Request& q) -> long long { return q.q_len > 0 ? blocks_of(q) + kItemUnits : 0; };
  auto work_of = [&](int i) -> long long { return i < p.R ? units_of_head(request_of(p, i)) * p.H_kv : 0; };
  auto take_share = [&](long long total) {
    share = Div::share(total, p.workgroups);
    at = share * blockIdx.x;
    end = min(at + share, total);
  };
  if (p.R <= kWave) {  // every wave for itself, nothing through LDS
    const Request mine = lane < p.R ? request_of(p, lane) : Request{0, 0, 0};
    const long long units = units_of_head(mine), w = units * p.H_kv, until = wave_scan(w);
    take_share(read_lane64(until, kWave - 1));
    if (at >= end) return;
    r = __builtin_ctzll(__ballot(at < until));
    rest = at - read_lane64(until - w, r);
    per_head = read_lane64(units, r);
    rq = mine.of_lane(r);
  } else {
    if (threadIdx.x < 2) found[threadIdx.x] = 0;
    long long total = 0;
    for (int base = 0; base < p.R; base += kThreads) total += block_sum<kThreads>(work_of(base + threadIdx.x), scan);
    take_share(total);
    if (at >= end) return;
    long long carry = 0;
    for (int base = 0; base < p.R && at >= carry; base += kThreads) {
      const long long w = work_of(base + threadIdx.x), before = carry + block_scan<kWaves>(w, lane, wave, scan, &carry);
      if (at >= before && at < before + w) {
        found[0] = base + threadIdx.x;
        found[1] = at - before;
      }
    }
    __syncthreads();
    r = __builtin_amdgcn_readfirstlane(static_cast<int>(found[0]));
    rest = read_lane64(found[1], 0);
    rq = request_of(p, r);
    per_head = units_of_head(rq);
  }
  int head = static_cast<int>(quotient(rest, per_head));
  rest -= head * per_head;

  while (true) {
    const int n_blocks = blocks_of(rq);
    const int b0 = max(static_cast<int>(rest) - kItemUnits, 0);
    const int b1 = static_cast<int>(min(rest + (end - at) - kItemUnits, static_cast<long long>(n_blocks)));
    if (b1 <= b0) return;  // only units that stand for no block are left
    const int rows = rq.q_len * p.G;

    // ---- queries: B operands, columns are query rows
    bf16x8 q[NC][kTerms][kSteps];
    int last_key[NC];  // last key that the column's row sees
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      const int in_tile = s * COLS + (PAIRED ? c & 7 : c);
      const bool exists = in_tile < rows;
      const int token = in_tile / p.G, h = in_tile - token * p.G;
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
    const int open = visible(rq, 0) / kKv4Block;

    floatx4 o[NC][kFrags], l[NC];  // l: sums of weights, by a product with ones; all four the same
    Reference ref[NC];
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      ref[s] = Reference{kLowest, p.scale_log2};
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
      wait_block<D>(i + 1 < mine);
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
        if (__any(top * ref[s].by > ref[s].m + kSlack)) {
          const float shrink = ref[s].raise(max_across_rows(top), p.scale_log2);
          l[s] *= shrink;
#pragma unroll
          for (int f = 0; f < kFrags; ++f) o[s][f] *= shrink;
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(z[s][e / 4][e % 4], ref[s].by, -ref[s].m));
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
        // and the outputs of the rows that do become NaN below (in other blocks all rows do, by the product).
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
        for (int s = 0; s < NC; ++s) {  // how many such tokens a row sees, of a chunk's channels
          uint32_t sees[4];
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const int key = key0 + e / 4 * 16 + 4 * kg + e % 4;
            sees[e / 2] = (key <= last_key[s] ? 0x3f80u : 0u) | (key < last_key[s] ? 0x3f800000u : 0u);
          }
          const floatx4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(n, words_to_bf16x8(sees[0], sees[1], sees[2], sees[3]),
                                                                     (floatx4{0.f, 0.f, 0.f, 0.f}), 0, 0, 0);
#pragma unroll
          for (int f = 0; f < kFrags; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[s][f][e] = hit[e] != 0.f ? NAN : o[s][f][e];
        }
      }
    }

    // ---- join the waves: every wave has read all of its ring
    float m[NC];
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      m[s] = passed_on(p, ref[s], last_key[s], table, b0 + wave, kWaves, b1);
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
        const RowOut<T> out(p, rq.first_row, head, row, top, sum);
        out.write(ch, x);
        if (ch == 0) out.write_lse();
      } else {
        *reinterpret_cast<float4*>(p.part_o + (part * ROWS + row) * D + ch) = x;
        if (ch == 0) p.part_ml[part * ROWS + row] = make_float2(top, sum);
      }
    }
    at += n_blocks + kItemUnits - rest;
    if (b0 == 0 && b1 < n_blocks) leave_item(p, blockIdx.x, rq, head, 0, rows, at - 1, share);
    if (at >= end) return;
    __syncthreads();
    // the next item
    rest = 0;
    if (++head == p.H_kv) {
      head = 0;
      do {
        if (++r >= p.R) return;
        rq = request_of(p, r);
      } while (rq.q_len == 0);
    }
  }
}

template <int D, typename T, int NC, bool PAIRED>
hipError_t launch(const AttnParams& p, hipStream_t s) {
  constexpr int rows = (PAIRED ? 8 : 16) * NC;
  kv4_attention_kernel<D, T, NC, PAIRED><<<p.workgroups, kThreads, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.workgroups == 1) return e;
  return launch_join<D, T, rows>(p, s);
}

}  // namespace

TileShape few_rows_shape(const Kv4AttentionArgs& a) {
  TileShape f;
  const long long most = min(static_cast<long long>(a.max_q_len) * a.G, static_cast<long long>(kFewRows));
  f.rows = most <= 8 ? 8 : most <= 16 ? 16 : 32;
  // Workgroups that run at once (a second round would have its first trips to memory by itself), and no more than can have
  // kMinUnits each.
  const long long longest = (static_cast<long long>(a.max_pages) << a.cache.page_shift) / kKv4Block;
  const double units = static_cast<double>(a.R) * a.H_kv * (longest + kItemUnits);
  f.workgroups = static_cast<int>(fmin(ceil(units / kMinUnits), static_cast<double>(kCus * workgroups_per_cu(a.dtype == SHOTKV_F32, f.rows))));
  return f;
}

template <int D>
static hipError_t launch_rows(const AttnParams& p, int dtype, int rows, hipStream_t s) {
  if (dtype == SHOTKV_F32) {
    if (rows == 8) return launch<D, float, 1, true>(p, s);
    return rows == 16 ? launch<D, float, 1, false>(p, s) : launch<D, float, 2, false>(p, s);
  }
  if (rows == 8) return launch<D, bf16_t, 1, true>(p, s);
  return rows == 16 ? launch<D, bf16_t, 1, false>(p, s) : launch<D, bf16_t, 2, false>(p, s);
}
hipError_t launch_few_rows(const AttnParams& p, int D, int dtype, int rows, hipStream_t s) {
  return D == 128 ? launch_rows<128>(p, dtype, rows, s) : launch_rows<64>(p, dtype, rows, s);
}

}  // namespace shotkv
