// Attention of many query rows per KV head over the paged 4-bit cache: chunks of prompts.
//
// A workgroup of four waves owns a tile of 128 (token, head) rows of one KV head, 32 to a wave, and walks the tokens that they
// see 64 at a time:
//   S^T = K Q^T      v_mfma_f32_32x32x16_bf16, tokens along the accumulator registers, query rows along the lanes, so maxima
//                    and sums of the softmax stay in the lane (and in the one 32 away).
//   O^T += V^T P^T   the same with channels along the registers: what a lane holds of the weights is its B operand.
// Codes become bf16 once per workgroup: every thread has one piece of 16 bytes of keys and one of values of the tokens after
// those that are worked on, converts them in the end of the step and puts them into the other half of the LDS, the values with
// tokens next to each other.  Products, weights and their two (fp32: three) bf16 numbers as in the kernel for few rows.
//
// Bound by the matrix cores and the power that they may take.  A weight of two numbers makes the second product twice as long:
// 24 matrix instructions per 32 tokens of 32 rows, of which the softmax sees 16, so 1.5 times the 4 D flops of a key and row.
// 2048 new tokens at the end of 32768 (32 heads over 8, 128 channels, bf16): 1365 to 1425 us by the card, 750 to 780 TFLOP/s of
// attention and 1130 to 1170 of matrix instructions, where the library's product of two 8192 x 8192 matrices has 1220.  64
// channels 545 TFLOP/s (as many weights per key, half the products), fp32 350.  Cache, queries and output, 69 MB, would take 14 us.
// Registers are full: the bf16 form of 128 channels spills 17 (72 bytes of scratch), and every form about 130 scalar ones into
// lanes of vector registers, most of them parameters that live through the loop.
// What was tried at that size: one number to a weight, a fifth faster but up to 2^-9 of a weight off; 64 rows to a wave, one
// wave to a SIMD, 2072 us; tiles of 256 rows with two groups of waves whose phases alternate, within 3% either way and 4% slower
// for 64 channels.
#include "kv4_attention.hpp"

namespace shotkv {

namespace {

typedef __attribute__((ext_vector_type(16))) float floatx16;
typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) u32x2 lds_u32x2;

constexpr int kStep = 64;  // tokens
constexpr int kRows = 128;  // of a tile
constexpr int kWaves = kRows / 32, kThreads = kWaves * kWave;
// An item's start and end take as long as some blocks do.  A workgroup has at least one step: 86 new tokens of 6106 with 4 heads
// over 4 take 29.6, 25.8 and 26.4 us with no less than 4, 6 and 8 units, five chunks of 63 of up to 368 17.9, 19.5 and 19.6.
constexpr int kItemUnits = 4, kMinUnits = 6;
typedef Division<kRows, kItemUnits, kMinUnits> Div;

// Waves to a SIMD: two, so that one multiplies while the other makes weights.  fp32 queries of 128 channels (and the three
// numbers that each is the sum of) do not fit into their 256 registers: two waves took 1890 us for 4 x 1024 new tokens of 4096
// with 32 heads over 8, most of it for spilled registers, one takes 735.
constexpr int waves_per_simd(int D, size_t bytes) { return D == 128 && bytes == 4 ? 1 : 2; }

// LDS of a step: keys [64][D], values [D][64], both in 16-byte columns that are swapped about within a row so that neither the
// writes nor the reads of a wave meet in a bank: column x of row r is at x ^ key_turn(r) and x ^ value_turn(r).
template <int D>
struct Stage {
  static constexpr int kKeyRow = D * 2, kValueRow = kStep * 2;
  static constexpr int kValues = kStep * kKeyRow;
  static constexpr int kBytes = kValues + D * kValueRow;
  static __device__ __forceinline__ uint32_t key_turn(uint32_t token) { return D == 128 ? token & 15 : (token >> 1) & 7; }
  static __device__ __forceinline__ uint32_t value_turn(uint32_t channel) { return ((channel >> 1) & 7) ^ ((channel >> 4) & 7); }
};

// A thread's piece of the codes of a step.
struct Piece {
  u32x4 k, v;
  uint32_t k_scale, v_scale;
  bool exists;  // the page that it came from
};

template <int D, typename T>
__global__ __launch_bounds__(kThreads, waves_per_simd(D, sizeof(T))) void kv4_prompt_kernel(AttnParams p) {
  typedef Kv4Block<D> B;
  typedef Stage<D> St;
  constexpr int kSteps = D / 16;                    // of the first product
  constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;    // bf16 numbers that a query element is the sum of
  constexpr int kNumbers = sizeof(T) == 4 ? 3 : 2;  // and a weight
  constexpr uint32_t kNotFinite = 1, kGone = 2;
  constexpr int kFrags = D / 32;                    // 32 channels each of the second product: groups of one scale
  __shared__ long long scan[kWaves + 1];
  __shared__ long long found[2];
  __shared__ __align__(256) char lds[2 * St::kBytes];
  static_assert(2 * St::kBytes >= kWaves / 2 * (kFrags * 16 + 2) * kWave * 4, "sums of half of the waves");
  // of four waves' tokens: kNotFinite, a value is not finite; kGone, the table names no page for them
  __shared__ __align__(16) uint32_t flags[2][4];
  __shared__ uint32_t scales[2][kStep / 4][D / 32];         // value scales, four tokens each
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = lane & 31, h = lane >> 5;

  // ---- this workgroup's share: the request, head and tile that hold its first unit
  auto units_of_head = [&](const Request& q, int tiles) { return read_lane64(wave_scan(Div::units(q, p.G, lane, tiles, kWave)), kWave - 1); };
  auto units_of = [&](const Request& q) -> long long {  // a lane's request, one head; a long one's by all lanes together
    const int tiles = Div::tiles(q, p.G);
    constexpr int kAlone = 2;
    long long mine = tiles <= kAlone ? Div::units(q, p.G, 0, tiles) : 0;
    for (unsigned long long left = __ballot(tiles > kAlone); left; left &= left - 1) {
      const int from = __builtin_ctzll(left);
      const Request other = q.of_lane(from);
      const long long sum = units_of_head(other, Div::tiles(other, p.G));
      if (lane == from) mine = sum;
    }
    return mine;
  };
  auto request = [&](int i) { return i < p.R ? request_of(p, i) : Request{0, 0, 0}; };
  long long at, end, share, rest, per_head;
  int me, r;
  Request rq;
  auto take_share = [&](long long total) {
    share = Div::share(total, p.workgroups);
    // Workgroups are dealt to the eight XCDs round-robin; neighbours, which read the same keys, go to one, whose L2 has them.
    constexpr int kXcds = 8;
    const int taken = static_cast<int>(quotient(total + share - 1, share)), xcd = blockIdx.x % kXcds;
    const bool idle = static_cast<int>(blockIdx.x) >= taken;
    me = idle ? blockIdx.x : xcd * (taken / kXcds) + min(xcd, taken % kXcds) + static_cast<int>(blockIdx.x) / kXcds;
    if (tid == 0) p.cut[me].rows = 0;
    at = share * me;
    end = min(at + share, total);
    return !idle;
  };
  if (p.R <= kWave) {  // every wave for itself, nothing through LDS
    const Request mine = request(lane);
    const long long units = units_of(mine), w = units * p.H_kv, until = wave_scan(w), total = read_lane64(until, kWave - 1);
    if (!take_share(total)) return;
    r = __builtin_ctzll(__ballot(at < until));
    rest = at - read_lane64(until - w, r);
    per_head = read_lane64(units, r);
    rq = mine.of_lane(r);
  } else {
    if (tid < 2) found[tid] = 0;
    long long total = 0;
    for (int base = 0; base < p.R; base += kThreads) total += block_sum<kThreads>(units_of(request(base + tid)) * p.H_kv, scan);
    if (!take_share(total)) return;
    long long carry = 0;
    for (int base = 0; base < p.R && at >= carry; base += kThreads) {
      const long long w = units_of(request(base + tid)) * p.H_kv, before = carry + block_scan<kWaves>(w, lane, wave, scan, &carry);
      if (at >= before && at < before + w) {
        found[0] = base + tid;
        found[1] = at - before;
      }
    }
    __syncthreads();
    r = __builtin_amdgcn_readfirstlane(static_cast<int>(found[0]));
    rest = read_lane64(found[1], 0);
    rq = request_of(p, r);
    per_head = units_of_head(rq, Div::tiles(rq, p.G));
  }
  int tiles = Div::tiles(rq, p.G);
  int head = static_cast<int>(quotient(rest, per_head)), tile = 0;
  rest -= head * per_head;
  for (long long carry = 0; tile < tiles; tile += kWave) {
    const long long until = carry + wave_scan(tile + lane < tiles ? Div::units(rq, p.G, tile + lane, tile + lane + 1) : 0);
    const unsigned long long after = __ballot(rest < until);
    if (after) {
      const int l = __builtin_ctzll(after);
      if (l) carry = read_lane64(until, l - 1);
      rest -= carry;
      tile += l;
      break;
    }
    carry = read_lane64(until, kWave - 1);
  }

  // ---- where this thread works
  const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
  // pieces: D = 128, every thread one of keys and one of values, D = 64, half of them each; waves 0 and 1 (0 and 2) have the
  // first block of the step
  const bool has_k = D == 128 || wave < 2, has_v = D == 128 || wave >= 2;
  const int half = D == 128 ? wave >> 1 : wave & 1, piece = D == 128 ? tid & 127 : tid & 63;
  const int k_token = 32 * half + piece / (D / 32), k_group = piece % (D / 32);
  const int v_quad = 8 * half + piece / (D / 8), v_chunk = piece % (D / 8);
  const uint32_t k_to = lds_base + k_token * St::kKeyRow, k_column = (4 * k_group) ^ St::key_turn(k_token);
  const int in_block = v_quad & 7;
  const uint32_t v_column = 4 * half + 2 * (in_block >> 2) + (in_block & 1);
  const uint32_t v_to = lds_base + St::kValues + v_chunk * 8 * St::kValueRow + ((in_block >> 1) & 1) * 8;
  const uint32_t v_turned = v_column ^ St::value_turn(8 * v_chunk);
  // operands
  // (column 2 j + h of a row is 32 j in the address of column h, by exclusive or: the rows are 128 or 256 bytes, and aligned)
  const uint32_t k_from = lds_base + n * St::kKeyRow + ((h ^ St::key_turn(n)) * 16);
  const uint32_t v_from = lds_base + St::kValues + n * St::kValueRow + ((h ^ St::value_turn(n)) * 16);
  uint32_t low = 0x0000bf80u, high = 0xbf800000u;
  asm("" : "+s"(low), "+s"(high));  // (as known constants they would become the inline -1.0, which is the high half for both)

  while (true) {
    const int n_blocks = Div::blocks(rq, p.G, tile);
    const int b0 = max(static_cast<int>(rest) - kItemUnits, 0);
    const int b1 = static_cast<int>(min(rest + (end - at) - kItemUnits, static_cast<long long>(n_blocks)));
    if (b1 <= b0) return;  // only units that stand for no block are left
    const int rows = min(rq.q_len * p.G - tile * kRows, kRows);
    // Up to 64 rows are two waves'; the other two then take the same rows, and every wave half of the tokens (16 requests of 4096
    // with 12 new tokens of 4 query heads to a KV head: 59 us, so 48.6).
    const bool split = rows <= kRows / 2;
    const int row_wave = split ? wave % (kWaves / 2) : wave;
    auto active = [&](int sub) { return row_wave * 32 < rows && (!split || wave / (kWaves / 2) == sub); };
    __syncthreads();  // the item before this one is done with the LDS

    // ---- queries
    bf16x8 q[kTerms][kSteps];
    const int row = row_wave * 32 + n;  // in the tile
    int limit;                      // last key that the lane's row sees in this range of blocks
    {
      const int flat = tile * kRows + row;
      const bool exists = row < rows;
      const int token = exists ? flat / p.G : 0, qh = exists ? flat - token * p.G : 0;
      limit = exists ? min(rq.len - rq.q_len + token, b1 * kKv4Block - 1) : -1;
      const char* src = p.q.token(rq.first_row + token) + (head * p.G + qh) * p.q.head_stride;
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        const int ch = 16 * j + 8 * h;
        if constexpr (sizeof(T) == 2) {
          q[0][j] = *reinterpret_cast<const bf16x8*>(src + ch * 2);
        } else {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = reinterpret_cast<const float*>(src)[ch + i];
#pragma unroll
          for (int t = 0; t < kTerms; ++t) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
              x[2 * i] -= low_half(w[i]);
              x[2 * i + 1] -= high_half(w[i]);
            }
            q[t][j] = words_to_bf16x8(w[0], w[1], w[2], w[3]);
          }
        }
      }
    }
    const int open = min(visible(rq, tile * kRows / p.G), b1 * kKv4Block);  // keys below are seen by all rows

    // Pages and pieces.
    const int32_t* table = p.block_table + static_cast<size_t>(r) * p.max_pages;
    const int page_shift = p.cache.page_shift - 5, in_page = (1 << page_shift) - 1;
    const long long page_bytes = static_cast<long long>(p.cache.H_kv << page_shift) * B::kBytes;
    const char* const head_base = p.cache.base + static_cast<long long>(head << page_shift) * B::kBytes;
    int pages = 0, first = -64;  // lane i: page of this wave's half of step first + i
    auto fetch = [&](int step, Piece& x) __attribute__((always_inline)) {
      if (step >= first + 64) {
        first = step;
        pages = table[min((b0 + 2 * (first + lane) + half) >> page_shift, p.max_pages - 1)];
      }
      const int page = __builtin_amdgcn_readlane(pages, step - first), blk = b0 + 2 * step + half;
      x.exists = page >= 0 && page < p.cache.n_pages && blk < b1;
      const char* base = head_base + (x.exists ? page : 0) * page_bytes + (blk & in_page) * B::kBytes;
      if (has_k) {
        x.k = *reinterpret_cast<const u32x4*>(base + B::kKeys + piece * 16);
        x.k_scale = *reinterpret_cast<const uint8_t*>(base + B::kKeyScales + piece);
      }
      if (has_v) {
        x.v = *reinterpret_cast<const u32x4*>(base + B::kValues + piece * 16);
        x.v_scale = *reinterpret_cast<const uint32_t*>(base + B::kValueScales + ((v_quad & 7) * (D / 32) + v_chunk / 4) * 4);
      }
    };
    auto put = [&](auto half_constant, int step, Piece& x) __attribute__((always_inline)) {  // into its half of the LDS
      constexpr int kHalf = decltype(half_constant)::value;
      constexpr uint32_t stage = kHalf * St::kBytes;
      if (has_k) {
        const float scale = kv4_scale(x.k_scale);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x4 w;
          w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.k[i], scale, 0));
          w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.k[i], scale, 1));
          w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.k[i], scale, 2));
          w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.k[i], scale, 3));
          *reinterpret_cast<lds_u32x4*>(static_cast<uintptr_t>(k_to + ((k_column ^ i) * 16)) + stage) = w;
        }
      }
      uint32_t any = 0;
      if (has_v) {
        const int token0 = (b0 + 2 * step) * kKv4Block + 4 * v_quad;
        if (!x.exists || token0 + 3 >= rq.len) {  // what lies past the request's tokens may be anything
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!x.exists || token0 + e >= rq.len) {
              x.v[e] = 0u;
              x.v_scale &= ~(0xffu << (8 * e));
            }
        }
        any = (((x.v_scale & 0x7f7f7f7fu) + 0x01010101u) & x.v_scale) & 0x80808080u;
        if (v_chunk % 4 == 0) scales[kHalf][v_quad][v_chunk / 4] = x.v_scale;
      }
      const bool not_finite = __any(any != 0);
      if (lane == 0) flags[kHalf][wave] = (not_finite ? kNotFinite : 0u) | (x.exists ? 0u : kGone);
      if (has_v) {
        if (not_finite) {  // (a NaN times no weight would reach the rows that do not see it)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if ((x.v_scale >> (8 * e) & 0xffu) == kKv4NotFinite) {
              x.v[e] = 0u;
              x.v_scale &= ~(0xffu << (8 * e));
            }
        }
        float scale[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)  // (the conversion looks at the exponent alone)
          scale[e] = __uint_as_float(e == 3 ? x.v_scale >> 1 : x.v_scale << (23 - 8 * e));
        auto pair = [&](auto constant) __attribute__((always_inline)) {
          constexpr int i = decltype(constant)::value;  // channels 2 i and 2 i + 1 of the chunk
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.v[e], scale[e], i));
          const uintptr_t to = static_cast<uintptr_t>(v_to + ((v_turned ^ i) * 16)) + stage + 2 * i * St::kValueRow;
          *reinterpret_cast<lds_u32x2*>(to) =
              u32x2{__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u)};
          *reinterpret_cast<lds_u32x2*>(to + St::kValueRow) =
              u32x2{__builtin_amdgcn_perm(w[1], w[0], 0x07060302u), __builtin_amdgcn_perm(w[3], w[2], 0x07060302u)};
        };
        pair(Constant<0>{});
        pair(Constant<1>{});
        pair(Constant<2>{});
        pair(Constant<3>{});
      }
    };

    floatx16 o[kFrags];
    Reference ref{kLowest, p.scale_log2};
    float l = 0.f;
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[f][e] = 0.f;

    bf16x8 v[2 * kFrags], w[kNumbers][2];  // values and weights of 32 tokens
    floatx16 z;                            // logits of 32 tokens
    u32x4 flagged{};                       // and the flags of their step
#pragma unroll
    for (int i = 0; i < 2 * kFrags; ++i) v[i] = words_to_bf16x8(0u, 0u, 0u, 0u);
#pragma unroll
    for (int t = 0; t < kNumbers; ++t) w[t][0] = w[t][1] = words_to_bf16x8(0u, 0u, 0u, 0u);
    auto gather = [&](int from, int to) __attribute__((always_inline)) {  // of the 2 * kFrags operands
#pragma unroll
      for (int i = from; i < to; ++i)
#pragma unroll
        for (int t = 0; t < kNumbers; ++t)
          o[i / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[i], w[t][i & 1], o[i / 2], 0, 0, 0);
    };
    // The two phases of 32 tokens.  First all products: the values of the 32 tokens before with their weights, then the logits.
    // Keys are asked for half by half, into the registers that the values leave.
    auto multiply = [&](auto half_constant, int sub) __attribute__((always_inline)) {
      constexpr int stage = decltype(half_constant)::value * St::kBytes;
      if (!active(sub)) return;
      bf16x8 k[kSteps];
      auto read_keys = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int j = from; j < to; ++j)
          k[j] = *reinterpret_cast<lds_bf16x8*>(static_cast<uintptr_t>(k_from ^ (32 * j)) + stage + sub * 32 * St::kKeyRow);
      };
      __builtin_amdgcn_s_setprio(1);
      read_keys(0, kSteps / 2);
      gather(0, kFrags);
      __builtin_amdgcn_sched_barrier(0);
      read_keys(kSteps / 2, kSteps);
      gather(kFrags, 2 * kFrags);
      __builtin_amdgcn_sched_barrier(0);
      flagged = *reinterpret_cast<const u32x4*>(flags[decltype(half_constant)::value]);
      z = floatx16{};
#pragma unroll
      for (int j = 0; j < kSteps; ++j)
#pragma unroll
        for (int t = 0; t < kTerms; ++t) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[j], q[t][j], z, 0, 0, 0);
      __builtin_amdgcn_s_setprio(0);
    };
    // Then the weights.
    auto weigh = [&](auto half_constant, int step, int sub) __attribute__((always_inline)) {
      constexpr int kHalf = decltype(half_constant)::value, stage = kHalf * St::kBytes;
      if (!active(sub)) return;
      const int key0 = (b0 + 2 * step) * kKv4Block;
      const uint32_t any = __builtin_amdgcn_readfirstlane(flagged[0] | flagged[1] | flagged[2] | flagged[3]);
      if (key0 + kStep > open || any & kGone) {
        const uint32_t mine = D == 128 ? (sub ? flagged[2] | flagged[3] : flagged[0] | flagged[1]) : (sub ? flagged[1] | flagged[3] : flagged[0] | flagged[2]);
        const int key = key0 + 32 * sub + 4 * h, most = mine & kGone ? -1 : limit;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (key + 8 * (e / 4) + e % 4 > most) z[e] = -INFINITY;
      }
      float top = z[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = __builtin_elementwise_maximum(top, z[e]);
      if (__any(top * ref.by > ref.m + kSlack)) {
        const float shrink = ref.raise(max_across_halves(top), p.scale_log2);
        l *= shrink;
#pragma unroll
        for (int f = 0; f < kFrags; ++f) o[f] *= shrink;
      }
      float x[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        x[e] = __builtin_amdgcn_exp2f(fmaf(z[e], ref.by, -ref.m));
        l += x[e];
      }
      if (any & kNotFinite) {
        // outputs of rows that see a value that is not finite
        const int left = limit - (key0 + 32 * sub + 4 * h);
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
          bool hit = false;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t word = scales[kHalf][8 * sub + 2 * i + h][f];
#pragma unroll
            for (int e = 0; e < 4; ++e) hit |= 8 * i + e <= left && (word >> (8 * e) & 0xffu) == kKv4NotFinite;
          }
          __builtin_amdgcn_sched_barrier(0);
          if (max_across_halves(hit ? 1.f : 0.f) > 0.f) {
#pragma unroll
            for (int e = 0; e < 16; ++e) o[f][e] = NAN;
          }
        }
      }
#pragma unroll
      for (int t = 0; t < kNumbers; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t words[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float &a = x[8 * i + 2 * e], &b = x[8 * i + 2 * e + 1];
            words[e] = pack_bf16(a, b);
            if (t + 1 < kNumbers) {
              a = less(a, words[e], low);
              b = less(b, words[e], high);
            }
          }
          w[t][i] = words_to_bf16x8(words[0], words[1], words[2], words[3]);
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int f = 0; f < kFrags; ++f)
#pragma unroll
        for (int i = 0; i < 2; ++i)  // columns 4 sub + 2 i + h of rows 32 f + n, whose turn differs from row n's by 2 f
          v[2 * f + i] = *reinterpret_cast<lds_bf16x8*>(static_cast<uintptr_t>(v_from ^ (32 * ((2 * sub + i) ^ f))) + stage + f * 32 * St::kValueRow);
    };
    const int steps = (b1 - b0 + 1) / 2;
    Piece next{};
    // A step on one half of the LDS, and the tokens after it into the other.
    auto work = [&](auto half_constant, int step) __attribute__((always_inline)) {
      constexpr Constant<decltype(half_constant)::value> here{};
      constexpr Constant<1 - decltype(half_constant)::value> there{};
      multiply(here, 0);
      weigh(here, step, 0);
      multiply(here, 1);
      weigh(here, step, 1);
      if (step + 1 < steps) {
        put(there, step + 1, next);
        if (step + 2 < steps) fetch(step + 2, next);
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
    };
    fetch(0, next);
    put(Constant<0>{}, 0, next);
    if (steps > 1) fetch(1, next);
    __syncthreads();
    for (int step = 0; step < steps; step += 2) {
      work(Constant<0>{}, step);
      if (step + 1 < steps) work(Constant<1>{}, step + 1);
    }
    if (row_wave * 32 < rows) gather(0, 2 * kFrags);
    float m = passed_on(p, ref, limit, table, b0 + (split ? wave / (kWaves / 2) : 0), split ? 2 : 1, b1);
    if (split) {  // the two halves of the tokens together, through the LDS that all are done with
      float* const sums = reinterpret_cast<float*>(lds) + (row_wave * (kFrags * 16 + 2)) * kWave + lane;
      if (wave >= kWaves / 2) {
        sums[0] = m;
        sums[kWave] = l;
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
#pragma unroll
          for (int e = 0; e < 16; ++e) sums[(2 + f * 16 + e) * kWave] = o[f][e];
      }
      __syncthreads();
      if (wave < kWaves / 2) {
        const float grown = fmaxf(m, sums[0]), mine = __builtin_amdgcn_exp2f(m - grown), other = __builtin_amdgcn_exp2f(sums[0] - grown);
        m = grown;
        l = l * mine + sums[kWave] * other;
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[f][e] = o[f][e] * mine + sums[(2 + f * 16 + e) * kWave] * other;
      }
    }

    // ---- a lane has four times four channels of every 32 of its row
    const bool whole = b0 == 0 && b1 == n_blocks;
    const size_t part = 2 * static_cast<size_t>(me) + (b0 == 0 ? 1 : 0);
    const float sum = sum_across_halves(l);
    if (row < rows && (!split || wave < kWaves / 2)) {
      if (whole) {
        const RowOut<T> out(p, rq.first_row, head, tile * kRows + row, m, sum);
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            out.write(32 * f + 8 * i + 4 * h, make_float4(o[f][4 * i], o[f][4 * i + 1], o[f][4 * i + 2], o[f][4 * i + 3]));
        if (h == 0) out.write_lse();
      } else {
        float* to = p.part_o + (part * kRows + row) * D + 4 * h;
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<float4*>(to + 32 * f + 8 * i) = make_float4(o[f][4 * i], o[f][4 * i + 1], o[f][4 * i + 2], o[f][4 * i + 3]);
        if (h == 0) p.part_ml[part * kRows + row] = make_float2(m, sum);
      }
    }
    at += n_blocks + kItemUnits - rest;
    if (b0 == 0 && b1 < n_blocks) leave_item(p, me, rq, head, tile, rows, at - 1, share);
    if (at >= end) return;
    // the next item
    rest = 0;
    if (++tile == tiles) {
      tile = 0;
      if (++head == p.H_kv) {
        head = 0;
        do {
          if (++r >= p.R) return;
          rq = request_of(p, r);
          tiles = Div::tiles(rq, p.G);
        } while (tiles == 0);
      }
    }
  }
}

template <int D, typename T>
hipError_t launch(const AttnParams& p, hipStream_t s) {
  kv4_prompt_kernel<D, T><<<p.workgroups, kThreads, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.workgroups == 1) return e;
  return launch_join<D, T, kRows>(p, s);
}

}  // namespace

int many_rows_at_once(const Kv4AttentionArgs& a) {
  return kCus * waves_per_simd(a.D, a.dtype == SHOTKV_F32 ? 4 : 2);  // a workgroup has a wave on every SIMD
}
TileShape many_rows_shape(const Kv4AttentionArgs& a) {
  const long long tiles = (static_cast<long long>(a.max_q_len) * a.G + kRows - 1) / kRows;
  const long long longest = (static_cast<long long>(a.max_pages) << a.cache.page_shift) / kKv4Block;
  const double units = static_cast<double>(a.R) * a.H_kv * tiles * (longest + kItemUnits);
  return TileShape{kRows, static_cast<int>(fmin(ceil(units / kMinUnits), many_rows_at_once(a)))};
}
hipError_t launch_many_rows(const AttnParams& p, int D, int dtype, hipStream_t s) {
  if (dtype == SHOTKV_F32) return D == 128 ? launch<128, float>(p, s) : launch<64, float>(p, s);
  return D == 128 ? launch<128, bf16_t>(p, s) : launch<64, bf16_t>(p, s);
}

}  // namespace shotkv
