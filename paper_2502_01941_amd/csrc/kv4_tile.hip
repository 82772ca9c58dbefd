// Attention of trees and windows, bf16, for tiles of 64 query rows per KV head over the paged 4-bit cache.
//
// The products, weights and layouts are those of the kernel for few rows (kv4_attention.hip): S^T = K Q^T and O^T += V^T P^T by
// v_mfma_f32_16x16x32_bf16, four sets of 16 rows to a tile.  Every wave of a workgroup takes blocks of 32 tokens in turn
// through a ring of its own, for all 64 rows: codes are converted once for four times 16 rows, and no wave waits for
// another until the end.  Queries are in LDS in the order of the operands; a wave's sums fill half of its registers, all of
// which are in use, so what the loop's addresses and masks follow from is made anew or read from LDS in it: one that is spilled would be
// read back behind the blocks in flight.  At the end the waves exchange sums in two rounds, after which each has those of one set
// of 16 rows, and writes them.
//
// Bound by matrix and vector instructions together, which overlap little here (beside the products of another wave a vector
// instruction takes 9.7 cycles, alone 4.3, measured): for 32 tokens of 64 rows 96 of the first (1540 cycles) and 400 of the second, 32 of them
// exponentials.  2048 new tokens of 32768 with a window of 4096 (32 heads over 8, 128 channels) 193 us, 1.07 PFLOP/s of products that
// are made for 0.72 of attention (weights of two numbers), the matrix cores busy for 42 % of the cycles at 2.2 GHz, vector instructions
// issued in another 44 %.  Two waves to a SIMD, of which the one that makes weights goes first (s_setprio), so that the other's products
// fill in: 16 requests of 4096 to 5120 tokens with 16 drafts each 49.8 us with the join, where waves of equal rank take 52.5 and waves whose
// products go first 52.0.  In such a call 20 us go by the tokens; a launch, the first blocks and three trips to memory before them are
// 7, exchange and output 4, the join and its launch 8, and workgroups that end before the last 5.
#include "kv4_blocks.hpp"

namespace shotkv {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kSets = 4, kRows = 16 * kSets;
// An item's start and end count for 16 blocks, and a workgroup has at least half as many units: 64 requests of 200 to 32768 tokens with
// 16 drafts take 177 us, with 7 units 202, with 4 233; 16 requests of 4096 to 5120 52, 55 and 56.
constexpr int kItemUnits = 16, kMinUnits = 8;
// Two blocks to a wave (three: 59.5 us for 57.3).
constexpr int kRingBlocks = 2;
typedef Division<kRows, kItemUnits, kMinUnits> Div;

constexpr int kWorkgroupsPerCu = 2;  // by registers and LDS

typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) u32x4 lds_piece;

// The lane's number, made anew: what follows from it is not kept in registers over a loop in which there are none to spare.
__device__ __forceinline__ int lane_again() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(lane));
  return lane;
}

template <int D, int SEEN>
__global__ __launch_bounds__(kThreads, kWorkgroupsPerCu) void kv4_tile_kernel(AttnParams p) {
  constexpr int kSteps = D / 32;  // of the first product
  constexpr int kNumbers = 2;     // bf16 numbers that a weight is the sum of
  constexpr int kFrags = D / 16;  // 16 channels each of the second product
  typedef Ring<D, kRingBlocks> R;
  constexpr int kRings = kWaves * R::kBytes, kQueries = kSets * kSteps * kWave * 16;
  constexpr int kSetBytes = kFrags * 4 * kWave * 4, kExchange = kWaves * 2 * kSetBytes;  // sums of a set; two sets of each wave
  __shared__ long long scan[kWaves + 1];
  __shared__ long long found[2];
  __shared__ float sh_m[kWaves][kRows], sh_l[kWaves][kRows];
  __shared__ int sh_first[kRows], sh_token[kRows];  // what a row's sight needs: see Sight
  __shared__ __align__(16) char lds[kRings + kQueries > kExchange ? kRings + kQueries : kExchange];
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c = lane & 15, kg = lane >> 4;
  const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
  const uint32_t ring = lds_base + wave * R::kBytes, queries = lds_base + kRings;

  uint32_t low = 0x0000bf80u, high = 0xbf800000u, two_ones = 0x3f803f80u;
  asm("" : "+s"(low), "+s"(high), "+s"(two_ones));  // (as known constants they would become the inline -1.0, which is the high half for both)

  // ---- this workgroup's share: the request, head and tile that hold its first unit
  auto units_of_head = [&](const Request& q, int tiles) { return read_lane64(wave_scan(Div::template units<SEEN>(p, q, lane, tiles, kWave)), kWave - 1); };
  auto units_of = [&](const Request& q) -> long long {  // a lane's request, one head; a long one's by all lanes together
    const int tiles = Div::tiles(q, p.G);
    constexpr int kAlone = 2;
    const bool alone = SEEN == kTree || tiles <= kAlone;
    long long mine = alone ? Div::template units<SEEN>(p, q, 0, tiles) : 0;
    for (unsigned long long left = __ballot(!alone); left; left &= left - 1) {
      const int from = __builtin_ctzll(left);
      const Request other = q.of_lane(from);
      const long long sum = units_of_head(other, Div::tiles(other, p.G));
      if (lane == from) mine = sum;
    }
    return mine;
  };
  auto request_number = [&](int i) { return i < p.R ? request_of<SEEN>(p, i) : Request{0, 0, 0, 0}; };
  long long at, end, share, rest, per_head;
  int me, r;
  Request rq;
  auto take_share = [&](long long total) {
    share = Div::share(total, p.workgroups);
    const int taken = static_cast<int>(quotient(total + share - 1, share));
    const bool idle = static_cast<int>(blockIdx.x) >= taken;
    me = idle ? blockIdx.x : in_xcd_order(blockIdx.x, taken);
    if (tid == 0) p.cut[me].rows = 0;
    at = share * me;
    end = min(at + share, total);
    return !idle;
  };
  int tiles, head, tile;
  if (p.whole) {
    const int most = (p.max_q_len * p.G + kRows - 1) / kRows, number = in_xcd_order(blockIdx.x, gridDim.x);
    tile = number % most;
    head = number / most % p.H_kv;
    r = number / most / p.H_kv;
    rq = request_of<SEEN>(p, r);
    tiles = Div::tiles(rq, p.G);
    if (tile >= tiles) return;
    me = 0;  // (it leaves no parts)
    at = rest = 0;
    end = share = Div::template units<SEEN>(p, rq, tile, tile + 1);
  } else {
    if (p.R <= kWave) {  // every wave for itself, nothing through LDS
      const Request mine = request_number(lane);
      const long long units = units_of(mine), w = units * p.H_kv, until = wave_scan(w), total = read_lane64(until, kWave - 1);
      if (!take_share(total)) return;
      r = __builtin_ctzll(__ballot(at < until));
      rest = at - read_lane64(until - w, r);
      per_head = read_lane64(units, r);
      rq = mine.of_lane(r);
    } else {
      if (tid < 2) found[tid] = 0;
      long long total = 0;
      for (int base = 0; base < p.R; base += kThreads) total += block_sum<kThreads>(units_of(request_number(base + tid)) * p.H_kv, scan);
      if (!take_share(total)) return;
      long long carry = 0;
      for (int base = 0; base < p.R && at >= carry; base += kThreads) {
        const long long w = units_of(request_number(base + tid)) * p.H_kv, before = carry + block_scan<kWaves>(w, lane, wave, scan, &carry);
        if (at >= before && at < before + w) {
          found[0] = base + tid;
          found[1] = at - before;
        }
      }
      __syncthreads();
      r = __builtin_amdgcn_readfirstlane(static_cast<int>(found[0]));
      rest = read_lane64(found[1], 0);
      rq = request_of<SEEN>(p, r);
      per_head = units_of_head(rq, Div::tiles(rq, p.G));
    }
    tiles = Div::tiles(rq, p.G);
    head = static_cast<int>(quotient(rest, per_head));
    tile = 0;
    rest -= head * per_head;
    for (long long carry = 0; tile < tiles; tile += kWave) {
      const long long until = carry + wave_scan(tile + lane < tiles ? Div::template units<SEEN>(p, rq, tile + lane, tile + lane + 1) : 0);
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
  }

  while (true) {
    const Walk walk = Div::template walk<SEEN>(p, rq, tile);
    const int n_blocks = walk.count;
    const int b0 = max(static_cast<int>(rest) - kItemUnits, 0);
    const int b1 = static_cast<int>(min(rest + (end - at) - kItemUnits, static_cast<long long>(n_blocks)));
    if (b1 <= b0) return;  // only units that stand for no block are left
    const int rows = min(rq.q_len * p.G - tile * kRows, kRows);
    const Open all_see = open_of<SEEN>(p, rq, Div::first_token(p.G, tile), Div::last_token(rq, p.G, tile));
    __syncthreads();  // the item before this one is done with the LDS

    auto query_piece = [&](int set, int j) {
      return reinterpret_cast<lds_piece*>(static_cast<uintptr_t>(queries + lane * 16 + (set * kSteps + j) * kWave * 16));
    };
    auto token_of = [&](int row) { return row < rows ? (tile * kRows + row) / p.G : -1; };
    // ---- queries on their way: wave s brings set s
    u32x4 piece[kSteps];
    {
      const int row = wave * 16 + c, token = max(token_of(row), 0), h = row < rows ? tile * kRows + row - token * p.G : 0;
      const char* src = p.q.token(rq.first_row + token) + (head * p.G + h) * p.q.head_stride + (D == 128 ? 64 * kg : 32 * kg);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) piece[j] = *reinterpret_cast<const u32x4*>(src + 16 * j);
    }
    // ---- blocks on their way
    const int32_t* table = p.block_table + static_cast<size_t>(r) * p.max_pages;
    const int page_shift = p.cache.page_shift - 5;
    int pages = 0;  // lane i: page of this wave's block number first + i
    int first = 0;
    auto page_of = [&](int i) {  // of the wave's block number i
      if ((i & 63) == 0) {
        first = i;
        pages = table[min(walk.block(b0 + wave + (first + lane) * kWaves) >> page_shift, p.max_pages - 1)];
        asm volatile("" : "+v"(pages));  // arrived: waited for here, and not, with all blocks in flight, at every use
      }
      return __builtin_amdgcn_readlane(pages, i & 63);
    };
    uint32_t nowhere = 0;  // bit i: the table names no page for the block in slot i of the ring
    auto request = [&](int i) {
      const int blk = walk.block(b0 + wave + i * kWaves), slot = i % R::kDepth;
      const int page = page_of(i);
      const bool exists = page >= 0 && page < p.cache.n_pages;
      nowhere = (nowhere & ~(1u << slot)) | (exists ? 0u : 1u << slot);
      // where this lane fetches from in a block: keys, values, scales
      const int lane = lane_again();
      const uint32_t straight = lane * 16, key_piece = (lane & 15) * 64 + (lane >> 4) * 16, word = D == 128 ? 4096 + lane * 4 : (lane & 31) * 4;
      request_block<D>(p.cache.base + kv4_block_offset<D>(p.cache, exists ? page : 0, head, blk & ((1 << page_shift) - 1)),
                       ring + slot * R::kSlot, key_piece, straight, word);
    };
    const int mine = (b1 - b0 - wave + kWaves - 1) / kWaves;  // blocks of this wave (may be none)
    for (int i = 0; i < min(mine, R::kDepth); ++i) request(i);

    // ---- queries into LDS, in the order of the operands
#pragma unroll
    for (int j = 0; j < kSteps; ++j) *query_piece(wave, j) = piece[j];
    if (tid < kRows) {
      const int token = token_of(tid);
      sh_first[tid] = Sight<SEEN>(p, rq, token, token >= 0).first;
      sh_token[tid] = token;
    }
    __syncthreads();

    auto sight = [&](int row) { return Sight<SEEN>(rq, sh_token[row], sh_first[row]); };
    floatx4 o[kSets][kFrags];
    float l[kSets];  // of this lane's tokens
    Reference ref[kSets];
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      ref[s] = Reference{kLowest, p.scale_log2};
      l[s] = 0.f;
#pragma unroll
      for (int f = 0; f < kFrags; ++f) o[s][f] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    for (int i = 0; i < mine; ++i) {
      const int blk = walk.block(b0 + wave + i * kWaves);
      const int key0 = blk * kKv4Block;
      const int slot = i % R::kDepth;
      const bool ok = !(nowhere >> slot & 1u), masked = !ok || !all_see.has(blk);
      wait_block<D, R::kDepth>(i + 1 < mine);
      const int lane = lane_again(), c = lane & 15, kg = lane >> 4;
      BlockData<D> b;
      read_block<D>(ring + slot * R::kSlot, lane, b);
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the slot is free again
      if (i + R::kDepth < mine) request(i + R::kDepth);

      // S^T: rows are tokens a * 16 + 4 kg + e
      floatx4 z[kSets][2];
#pragma unroll
      for (int s = 0; s < kSets; ++s) z[s][0] = z[s][1] = floatx4{0.f, 0.f, 0.f, 0.f};
      const float key_scale[2] = {kv4_scale(b.ks[0]), kv4_scale(b.ks[1])};
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        const bf16x8 row[2] = {decode_word(b.k[0][j], key_scale[0]), decode_word(b.k[1][j], key_scale[1])};
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
          const bf16x8 q = *reinterpret_cast<lds_bf16x8*>(static_cast<uintptr_t>(queries + lane * 16 + (s * kSteps + j) * kWave * 16));
#pragma unroll
          for (int a = 0; a < 2; ++a) z[s][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(row[a], q, z[s][a], 0, 0, 0);
        }
      }
      uint32_t seen[kSets];     // in masked blocks: bit a * 16 + e, key a * 16 + 4 kg + e
      bool not_finite = false;  // values that are not and that some row must not see
      if (masked) {
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
          seen[s] = ok ? sight(s * 16 + c).word(p, rq, key0) >> (4 * kg) : 0u;
#pragma unroll
          for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!(seen[s] >> (a * 16 + e) & 1u)) z[s][a][e] = -INFINITY;
        }
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
          any |= may_not_be_finite<SEEN>(b.vs[a]);
        }
        not_finite = __any(any != 0);
      }

      __builtin_amdgcn_s_setprio(1);
      // weights
      bf16x8 w[kSets][kNumbers];
#pragma unroll
      for (int s = 0; s < kSets; ++s) {
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
#pragma unroll
        for (int t = 0; t < kNumbers; ++t) {
          uint32_t words[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            words[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
            l[s] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, words[e]), __builtin_bit_cast(bf16x2, two_ones), l[s], false);
            if (t + 1 < kNumbers) {
              x[2 * e] = less(x[2 * e], words[e], low);
              x[2 * e + 1] = less(x[2 * e + 1], words[e], high);
            }
          }
          w[s][t] = words_to_bf16x8(words[0], words[1], words[2], words[3]);
        }
      }

      // O^T
      float scale[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)  // (the conversion looks at the exponent alone: what is beside the byte does not matter)
        scale[e] = __uint_as_float(e % 4 == 3 ? b.vs[e / 4] >> 1 : b.vs[e / 4] << (23 - 8 * (e % 4)));
      if (not_finite) {
        // A NaN or an infinity in a product of zero weight would reach the rows that do not see its token: it is taken out of the
        // values, and the outputs of the rows that do become NaN below (in other blocks all rows do, by the product).
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (is_not_finite<SEEN>(b.v[e / 4][e % 4], (b.vs[e / 4] >> (8 * (e % 4))) & 0xffu)) {
            b.v[e / 4][e % 4] = 0u;
            scale[e] = 1.f;
            b.vs[e / 4] |= kKv4NotFinite << (8 * (e % 4));
          }
      }
      __builtin_amdgcn_s_setprio(0);
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
          for (int t = 0; t < kNumbers; ++t)
#pragma unroll
            for (int s = 0; s < kSets; ++s) o[s][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[s][t], o[s][f], 0, 0, 0);
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
        for (int s = 0; s < kSets; ++s) {  // how many such tokens a row sees, of a chunk's channels
          uint32_t sees[4];
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const int bit = e / 4 * 16 + e % 4;
            sees[e / 2] = (seen[s] >> bit & 1u ? 0x3f80u : 0u) | (seen[s] >> bit & 2u ? 0x3f800000u : 0u);
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

    // ---- the waves' references, then their sums: in two rounds, after which wave s has those of set s
    float m[kSets];
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      m[s] = passed_on<SEEN>(p, rq, ref[s], sight(s * 16 + c), walk, table, b0 + wave, kWaves, b1);
      if (kg == 0) sh_m[wave][s * 16 + c] = m[s];
    }
    __syncthreads();  // every wave has read all of its ring, and of the queries
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      const int row = s * 16 + c;
      float all = sh_m[0][row];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) all = fmaxf(all, sh_m[i][row]);
      const float shrink = __builtin_amdgcn_exp2f(m[s] - all);
      const float weights = sum_across_halves(sum_across_row_pairs(l[s])) * shrink;
      if (kg == 0) sh_l[wave][row] = weights;
#pragma unroll
      for (int f = 0; f < kFrags; ++f) o[s][f] *= shrink;
    }
    typedef __attribute__((address_space(3))) floatx4 lds_floatx4;
    auto place = [&](int w, int half, int f) {  // of four of this lane's sums, in the half of wave w
      return reinterpret_cast<lds_floatx4*>(static_cast<uintptr_t>(lds_base + (w * 2 + half) * kSetBytes + (f * kWave + lane) * 16));
    };
    floatx4 two[2][kFrags], one[kFrags];  // sets 2 (wave / 2) and the one after; set `wave`
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        const bool upper = wave >= 2;
        *place(wave, half, f) = upper ? o[half][f] : o[2 + half][f];
        two[half][f] = upper ? o[2 + half][f] : o[half][f];
      }
    __syncthreads();
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int f = 0; f < kFrags; ++f) two[half][f] += *place(wave ^ 2, half, f);
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {  // (into what this wave alone has read)
      *place(wave ^ 2, 0, f) = wave & 1 ? two[0][f] : two[1][f];
      one[f] = wave & 1 ? two[1][f] : two[0][f];
    }
    __syncthreads();
#pragma unroll
    for (int f = 0; f < kFrags; ++f) one[f] += *place(wave ^ 3, 0, f);

    const bool whole = b0 == 0 && b1 == n_blocks;
    const size_t part = 2 * static_cast<size_t>(me) + (b0 == 0 ? 1 : 0);
    {
      const int row = wave * 16 + c;
      float sum = 0.f, top = sh_m[0][row];
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        sum += sh_l[i][row];
        top = fmaxf(top, sh_m[i][row]);
      }
      if constexpr (D == 64) {
        // Lanes kg < 2 have the even channels of their chunks, the others the odd ones of the same: of the chunks e and e + 2
        // the lower half of the wave takes the first and the upper the second.
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(one[f][e]), __float_as_uint(one[f][e + 2]), false, false);
            one[f][e] = __uint_as_float(x[0]);
            one[f][e + 2] = __uint_as_float(x[1]);
          }
      }
      if (row < rows) {
        // eight channels each: four times (of 64: twice)
        auto each = [&](auto write) {
#pragma unroll
          for (int e = 0; e < (D == 128 ? 4 : 2); ++e) {
            if constexpr (D == 128) {
              write(8 * (4 * kg + e), make_float4(one[0][e], one[1][e], one[2][e], one[3][e]));
              write(8 * (4 * kg + e) + 4, make_float4(one[4][e], one[5][e], one[6][e], one[7][e]));
            } else {
              const int chunk = 4 * (kg & 1) + e + 2 * (kg >> 1);
              write(8 * chunk, make_float4(one[0][e], one[0][e + 2], one[1][e], one[1][e + 2]));
              write(8 * chunk + 4, make_float4(one[2][e], one[2][e + 2], one[3][e], one[3][e + 2]));
            }
          }
        };
        if (whole) {
          const RowOut<bf16_t> out(p, rq.first_row, head, tile * kRows + row, top, sum);
          each([&](int ch, const float4& x) { out.write(ch, x); });
          if (kg == 0) out.write_lse();
        } else {
          float* to = p.part_o + (part * kRows + row) * D;
          each([&](int ch, const float4& x) { *reinterpret_cast<float4*>(to + ch) = x; });
          if (kg == 0) p.part_ml[part * kRows + row] = make_float2(top, sum);
        }
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
          rq = request_of<SEEN>(p, r);
          tiles = Div::tiles(rq, p.G);
        } while (tiles == 0);
      }
    }
  }
}

template <int D, int SEEN>
hipError_t launch(const AttnParams& p, hipStream_t s) {
  kv4_tile_kernel<D, SEEN><<<p.workgroups, kThreads, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.workgroups == 1 || p.whole) return e;
  return launch_join<D, bf16_t, kRows>(p, s);
}

}  // namespace

// In us cut and whole, 32 heads over 8, 128 channels: 64 new tokens of 8192 to a request (32 items), a window of 500 (20 blocks), 4 requests 28
// and 19, 8 35 and 20, 16 50 and 28, 30 71 and 50; of 2000 (66), 3 33 and 40, 6 46 and 41, 16 80 and 58, 18 90 and 92, 30 134 and
// 110.  Trees of 16 drafts (8 items) over up to 300, one request 17 and 15, 32 25 and 16; up to 1000, one 17 and 24, 8 23 and 24, 32 34
// and 25, of lengths from 40 on 28 and 24; of lengths from 40 to 1500, 16 25 and 29, 32 30 and 31, 64 40 and 38; to
// 2000 (62 blocks), 32 32 and 36.
constexpr WholeItems kWholeWindows = {0.33, 18, 60, 72}, kWholeTrees = {0.33, 18, 45, 48};
TileShape tiles_of_64_shape(const Kv4AttentionArgs& a) {
  const long long tiles = (static_cast<long long>(a.max_q_len) * a.G + kRows - 1) / kRows;
  const double longest = longest_walk(a, a.seen == kTree ? a.max_q_len : kRows / a.G + 1);
  const double units = static_cast<double>(a.R) * a.H_kv * tiles * (longest + kItemUnits);
  return TileShape{kRows, static_cast<int>(fmin(ceil(units / kMinUnits), kCus * kWorkgroupsPerCu)),
                   whole_items(a, kRows, longest, a.seen == kTree ? kWholeTrees : kWholeWindows)};
}
hipError_t launch_tiles_of_64(const AttnParams& p, int seen, int D, hipStream_t s) {
  if (D == 64) return launch<64, kTree>(p, s);
  return seen == kWindow ? launch<128, kWindow>(p, s) : launch<128, kTree>(p, s);
}

}  // namespace shotkv
