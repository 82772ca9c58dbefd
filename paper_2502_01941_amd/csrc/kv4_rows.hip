// Rows of queries, keys and values on their way to attention: per-head norms and rotation in one pass, with the keys and
// values of new tokens going straight into the 4-bit cache, and the cache's writer and reader on their own.
//
// All of it moves rows and does some ten operations per value, so memory is the bound.  A lane holds eight channels of one
// row (16 bytes of bf16), D / 8 lanes a row, so a wave has four rows of 128 channels (eight of 64): the same head of
// consecutive tokens, which in a block of the cache are one piece of 256 bytes of value codes.  Sums of squares, partners
// of the rotation and the largest magnitude of a group of 32 channels are then exchanges between lanes of a row, and the
// angles of a token stay in registers while a wave goes through the heads.
//
// Measured, where a kernel that adds one to 1 GiB has 6.2 TB/s read and written and a copy 4.9: norms and rotation of 32768
// tokens of 32 + 8 heads of 128 in bf16, 671 MB, 140 us, 4.8 TB/s; of 16384 tokens with 64 channels 28 us, 6.1; 4001 tokens in
// fp32, 64 channels, 82 MB, 16 us, 5.1; 16 tokens that are stored as well 4 us, a launch and three trips to memory.  419328
// rows of 8 heads of 128 in bf16, 2.17 GB: 372 us to store (5.8 TB/s), 423 to load (5.1).
#include "kv4.hpp"

namespace shotkv {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
// Workgroups of norm_rope: enough to keep the chip full (2048: 16384 tokens with 64 channels 30 us, 4096: 28); enough for every
// CU to have its part.
constexpr int kEnough = 4096, kSome = 1024;

// Eight channels as they are in memory.
template <typename T>
struct RawRow {
  u32x4 w[sizeof(T) / 2];
};
// STREAM: past the caches, for rows that nobody reads again (the 419328 rows: 848 us stored and loaded without, 806 with).
template <typename T, bool STREAM = false>
__device__ __forceinline__ RawRow<T> fetch8(const char* p) {
  RawRow<T> r;
#pragma unroll
  for (unsigned i = 0; i < sizeof(T) / 2; ++i) {
    const u32x4* src = reinterpret_cast<const u32x4*>(p) + i;
    r.w[i] = STREAM ? __builtin_nontemporal_load(src) : *src;
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void widen8(const RawRow<T>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      x[2 * i] = __uint_as_float(r.w[0][i] << 16);
      x[2 * i + 1] = __uint_as_float(r.w[0][i] & 0xffff0000u);
    } else {
      x[i] = __uint_as_float(r.w[0][i]);
      x[4 + i] = __uint_as_float(r.w[1][i]);
    }
  }
}
template <typename T>
__device__ __forceinline__ void load8(const char* p, float (&x)[8]) { widen8<T>(fetch8<T>(p), x); }
typedef __attribute__((ext_vector_type(2))) float floatx2;
typedef __attribute__((ext_vector_type(4))) float floatx4;
__device__ __forceinline__ uint32_t to_bf16x2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{a, b}), bf16x2));
}
// Eight channels of a row whose lanes all store theirs.
template <typename T>
__device__ __forceinline__ void store8(char* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    __builtin_nontemporal_store(u32x4{to_bf16x2(x[0], x[1]), to_bf16x2(x[2], x[3]), to_bf16x2(x[4], x[5]), to_bf16x2(x[6], x[7])},
                                reinterpret_cast<u32x4*>(p));
  } else {
    // Four lanes of a row exchange their 128 bytes, so that each of the two instructions writes whole pieces of 64 (of every
    // lane's 32 the first and then the second half: 35100 rows of 8 heads of 128 are loaded in 109 us, so in 80).
    const bool odd = threadIdx.x & 1;
    floatx4 first, second;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t low = __float_as_uint(x[i]), high = __float_as_uint(x[4 + i]);
      const uint32_t low_a = __builtin_amdgcn_update_dpp(0u, low, 0x50, 0xf, 0xf, false);  // quad_perm [0,0,1,1]
      const uint32_t high_a = __builtin_amdgcn_update_dpp(0u, high, 0x50, 0xf, 0xf, false);
      const uint32_t low_b = __builtin_amdgcn_update_dpp(0u, low, 0xfa, 0xf, 0xf, false);  // quad_perm [2,2,3,3]
      const uint32_t high_b = __builtin_amdgcn_update_dpp(0u, high, 0xfa, 0xf, 0xf, false);
      first[i] = __uint_as_float(odd ? high_a : low_a);
      second[i] = __uint_as_float(odd ? high_b : low_b);
    }
    p -= (threadIdx.x & 3) * 16;
    __builtin_nontemporal_store(first, reinterpret_cast<floatx4*>(p));
    __builtin_nontemporal_store(second, reinterpret_cast<floatx4*>(p + 64));
  }
}
// To the nearest value of the storage type.
template <typename T>
__device__ __forceinline__ void round8(float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const uint32_t r = to_bf16x2(x[i], x[i + 1]);
      x[i] = __uint_as_float(r << 16);
      x[i + 1] = __uint_as_float(r & 0xffff0000u);
    }
  }
}

// A row of keys (or values) into its slot.
template <int D, bool VALUE>
__device__ __forceinline__ void put_row(const Kv4Pages& c, uint32_t slot, int head, int chunk, bool live, const float (&x)[8]) {
  uint32_t scale;
  const uint32_t codes = kv4_encode(x, &scale);  // by all lanes: rows of one wave exchange among themselves
  if (!live) return;
  typedef Kv4Block<D> B;
  char* block = kv4_block_of_slot<D>(c, slot, head);
  const int token = slot & 31;
  *reinterpret_cast<uint32_t*>(block + (VALUE ? B::value_word(token, chunk) : B::key_word(token, chunk))) = codes;
  if (chunk % 4 == 0)
    block[VALUE ? B::value_scale(token, chunk / 4) : B::key_scale(token, chunk / 4)] = static_cast<char>(scale);
}

constexpr int batch_of(int size) { return 8 / size; }  // rows of a type that are on their way together
// Where the other channel of a pair is: next to it; half a row away; half the turning channels away.
enum Pairs { kNeighbours, kHalves, kPartHalves };
// The four waves of a workgroup take neighbouring tokens, so that the rows that they read and write together are 4 KB in a
// layout by head.  Every wave goes through the heads [heads_per_group * blockIdx.y, + heads_per_group) of query, key and value
// heads in a row, one kind after the other with its weights in the angles, four rows (fp32: two) on their way together.  The
// pairs and the storing are constants: with all of them in one kernel its code alone took longer to fetch than 2000 tokens
// take (12 us for 8).  Asked for a row ahead instead of four at a time 32768 tokens took 161 us, with a head per wave of the
// same four tokens 177, with angles and weights read again for every head 435.
template <int D, typename T, Pairs PAIRS, bool STORES>
__global__ __launch_bounds__(kThreads, 5) void norm_rope_kernel(RopeArgs a, int heads_per_group) {
  constexpr int kLanes = D / 8, kRows = kWave / kLanes, kBatch = batch_of(sizeof(T));
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int chunk = lane % kLanes, c0 = chunk * 8;
  const int t = (blockIdx.x * kWaves + wave) * kRows + lane / kLanes;
  const bool in_batch = t < a.T;
  const int tc = min(t, a.T - 1);
  const int pos = a.token_pos[tc];
  const bool live = in_batch && pos >= 0 && pos < a.n_positions, all_live = __all(live);
  int slot = -1;
  if (STORES && live) slot = a.slot_map[tc];
  const bool stored = STORES && static_cast<uint32_t>(slot) < a.cache.n_slots;
  const int half = PAIRS == kHalves ? D / 2 : a.rot_dim / 2;
  const float* const angles = a.table + static_cast<size_t>(live ? pos : 0) * a.rot_dim;
  const bool turns = PAIRS == kHalves || c0 < a.rot_dim;
  const int partner = !turns || PAIRS == kNeighbours ? lane : c0 < half ? lane + half / 8 : lane - half / 8;

  const int keys_end = a.H + a.H_kv, all = keys_end + (STORES ? a.H_kv : 0);
  const int h_end = min(all, (static_cast<int>(blockIdx.y) + 1) * heads_per_group);
  for (int h = blockIdx.y * heads_per_group; h < h_end;) {  // one kind of heads after the other
    const bool is_q = h < a.H, is_v = STORES && h >= keys_end;
    const int first = is_q ? 0 : is_v ? keys_end : a.H, stop = min(h_end, is_q ? a.H : is_v ? all : keys_end);
    const RowView& in = is_q ? a.q : is_v ? a.v : a.k;
    const RowView& out = is_q ? a.q_out : a.k_out;
    const char* const src = in.token(tc) + c0 * sizeof(T);
    char* const dst = !is_v && out.data ? out.token(tc) + c0 * sizeof(T) : nullptr;
    RawRow<T> rows[kBatch];
    auto fetch = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) rows[i] = fetch8<T>(src + (min(h + i, stop - 1) - first) * in.head_stride);
    };
    fetch();
    // Of a pair's channels i and j, y[i] = inv * (x[i] * co[i] + x[j] * si[i]): cosine and signed sine times the norm's weights.
    const void* const weights = is_q ? a.q_weight : is_v ? nullptr : a.k_weight;
    float co[8], si[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      co[i] = 1.f;
      si[i] = 0.f;
    }
    if (turns && !is_v) {
      const floatx4* c = reinterpret_cast<const floatx4*>(angles + (PAIRS == kNeighbours ? c0 / 2 : c0 < half ? c0 : c0 - half));
      const floatx4* s = reinterpret_cast<const floatx4*>(reinterpret_cast<const float*>(c) + half);
      if constexpr (PAIRS == kNeighbours) {
        const floatx4 cosine = *c, sine = *s;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          co[2 * i] = co[2 * i + 1] = cosine[i];
          si[2 * i] = -sine[i];
          si[2 * i + 1] = sine[i];
        }
      } else {
        const floatx4 cosine[2] = {c[0], c[1]}, sine[2] = {s[0], s[1]};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          co[i] = cosine[i / 4][i % 4];
          si[i] = c0 < half ? -sine[i / 4][i % 4] : sine[i / 4][i % 4];
        }
      }
    }
    if (weights) {
      float own[8], other[8];
      load8<T>(static_cast<const char*>(weights) + c0 * sizeof(T), own);
      load8<T>(static_cast<const char*>(weights) + (c0 + (partner - lane) * 8) * static_cast<int>(sizeof(T)), other);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        co[i] *= own[i];
        si[i] *= PAIRS == kNeighbours ? other[i ^ 1] : other[i];
      }
    }
    auto work = [&](int head, const RawRow<T>& raw) __attribute__((always_inline)) {
      float x[8], y[8];
      widen8<T>(raw, x);
      if (is_v) {
        put_row<D, true>(a.cache, slot, head, chunk, stored, x);
        return;
      }
      float inv = 1.f;
      if (weights) {
        auto mean_square = [&]() __attribute__((always_inline)) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
          sum += __uint_as_float(lane_xor<1>(__float_as_uint(sum)));
          sum += __uint_as_float(lane_xor<2>(__float_as_uint(sum)));
          sum += __uint_as_float(lane_xor<4>(__float_as_uint(sum)));
          if (D == 128) sum += __uint_as_float(lane_xor<8>(__float_as_uint(sum)));
          return sum * (1.f / D);
        };
        const float square = mean_square() + a.eps;
        inv = rsqrtf(square);
        if (__any(!(square > 0x1p-100f && square < 0x1p120f))) {  // past what squares of 32 bits hold: once more, of other units
          const float by = square < 0x1p-100f ? 0x1p100f : square < 0x1p120f ? 1.f : 0x1p-70f;
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= by;
          inv = rsqrtf(mean_square() + a.eps * by * by);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float other = PAIRS == kNeighbours ? x[i ^ 1] : PAIRS == kHalves ? __uint_as_float(lane_xor<D / 16>(__float_as_uint(x[i]))) : __shfl(x[i], partner);
        y[i] = (turns ? fmaf(x[i], co[i], other * si[i]) : x[i] * co[i]) * inv;
      }
      if (!all_live) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = live ? y[i] : 0.f;
      }
      if (in_batch && dst) store8<T>(dst + head * out.head_stride, y);
      if (STORES && !is_q) {
        round8<T>(y);
        put_row<D, false>(a.cache, slot, head, chunk, stored, y);
      }
    };
    while (true) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (h + i < stop) work(h + i - first, rows[i]);
      h += kBatch;
      if (h >= stop) break;
      fetch();
    }
    h = stop;
  }
}

template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kv4_store_kernel(Kv4RowArgs a) {
  constexpr int kLanes = D / 8, kRows = kWave / kLanes;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int chunk = lane % kLanes;
  const int t = blockIdx.x * kRows + lane / kLanes;
  const int tc = min(t, a.T - 1);
  const int slot = a.slot_map[tc];
  const bool stored = t < a.T && static_cast<uint32_t>(slot) < a.cache.n_slots;
  const char* k = a.k.token(tc) + chunk * 8 * sizeof(T);
  const char* v = a.v.token(tc) + chunk * 8 * sizeof(T);
  for (int h = wave; h < a.cache.H_kv; h += kWaves) {
    float x[8], y[8];
    if (stored) {
      widen8<T>(fetch8<T, true>(k + h * a.k.head_stride), x);
      widen8<T>(fetch8<T, true>(v + h * a.v.head_stride), y);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = y[i] = 0.f;
    }
    put_row<D, false>(a.cache, slot, h, chunk, stored, x);
    put_row<D, true>(a.cache, slot, h, chunk, stored, y);
  }
}

template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kv4_load_kernel(Kv4RowArgs a) {
  constexpr int kLanes = D / 8, kRows = kWave / kLanes;
  typedef Kv4Block<D> B;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int chunk = lane % kLanes;
  const int t = blockIdx.x * kRows + lane / kLanes;
  if (t >= a.T) return;
  const int slot = a.slot_map[t];
  const bool stored = static_cast<uint32_t>(slot) < a.cache.n_slots;
  const int token = slot & 31;
  char* k = a.k.token(t) + chunk * 8 * sizeof(T);
  char* v = a.v.token(t) + chunk * 8 * sizeof(T);
  for (int h = wave; h < a.cache.H_kv; h += kWaves) {
    float x[8] = {}, y[8] = {};
    if (stored) {
      const char* block = kv4_block_of_slot<D>(a.cache, slot, h);
      kv4_decode(*reinterpret_cast<const uint32_t*>(block + B::key_word(token, chunk)),
                 kv4_scale(static_cast<uint8_t>(block[B::key_scale(token, chunk / 4)])), x);
      kv4_decode(*reinterpret_cast<const uint32_t*>(block + B::value_word(token, chunk)),
                 kv4_scale(static_cast<uint8_t>(block[B::value_scale(token, chunk / 4)])), y);
    }
    store8<T>(k + h * a.k.head_stride, x);
    store8<T>(v + h * a.v.head_stride, y);
  }
}

template <int D, typename T, Pairs PAIRS>
void launch_stores(const RopeArgs& a, const dim3& grid, int per_group, hipStream_t s) {
  if (a.cache.base) norm_rope_kernel<D, T, PAIRS, true><<<grid, kThreads, 0, s>>>(a, per_group);
  else norm_rope_kernel<D, T, PAIRS, false><<<grid, kThreads, 0, s>>>(a, per_group);
}
template <int D, typename T>
void launch_pairs(const RopeArgs& a, const dim3& grid, int per_group, hipStream_t s) {
  if (a.interleaved) launch_stores<D, T, kNeighbours>(a, grid, per_group, s);
  else if (a.rot_dim == D) launch_stores<D, T, kHalves>(a, grid, per_group, s);
  else launch_stores<D, T, kPartHalves>(a, grid, per_group, s);
}

}  // namespace

hipError_t launch_norm_rope(const RopeArgs& a, hipStream_t s) {
  const int tokens = kWave / (a.D / 8);  // of a wave
  // A wave keeps its tokens' angles through the heads that it goes through: all of them where that leaves enough workgroups,
  // fewer in short batches, but no part of what it has on its way together where all CUs have some without that (2000 tokens:
  // two heads to a wave 10.4 us, four 7.9).
  const int all = a.H + a.H_kv + (a.cache.base ? a.H_kv : 0);
  const int quads = ceil_div(a.T, tokens * kWaves), batch = batch_of(a.dtype == SHOTKV_BF16 ? 2 : 4);
  int per_group = ceil_div(all, min(ceil_div(kEnough, quads), all));
  if (static_cast<long long>(quads) * ceil_div(all, batch) >= kSome) per_group = ceil_div(per_group, batch) * batch;
  const dim3 grid(quads, ceil_div(all, per_group));
  if (a.D == 128) {
    if (a.dtype == SHOTKV_BF16) launch_pairs<128, bf16_t>(a, grid, per_group, s);
    else launch_pairs<128, float>(a, grid, per_group, s);
  } else {
    if (a.dtype == SHOTKV_BF16) launch_pairs<64, bf16_t>(a, grid, per_group, s);
    else launch_pairs<64, float>(a, grid, per_group, s);
  }
  return hipGetLastError();
}

#define SHOTKV_KV4_ROWS(kernel)                                                                    \
  const dim3 grid(ceil_div(a.T, kWave / (a.D / 8)));                                               \
  if (a.D == 128) {                                                                                \
    if (a.dtype == SHOTKV_BF16) kernel<128, bf16_t><<<grid, kThreads, 0, s>>>(a);                  \
    else kernel<128, float><<<grid, kThreads, 0, s>>>(a);                                          \
  } else {                                                                                         \
    if (a.dtype == SHOTKV_BF16) kernel<64, bf16_t><<<grid, kThreads, 0, s>>>(a);                   \
    else kernel<64, float><<<grid, kThreads, 0, s>>>(a);                                           \
  }                                                                                                \
  return hipGetLastError()

hipError_t launch_kv4_store(const Kv4RowArgs& a, hipStream_t s) { SHOTKV_KV4_ROWS(kv4_store_kernel); }
hipError_t launch_kv4_load(const Kv4RowArgs& a, hipStream_t s) { SHOTKV_KV4_ROWS(kv4_load_kernel); }

#undef SHOTKV_KV4_ROWS

}  // namespace shotkv
