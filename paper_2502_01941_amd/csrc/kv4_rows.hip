// Rows of queries, keys and values on their way to attention: per-head norms and rotation in one pass, with the keys and
// values of new tokens going straight into the 4-bit cache, and the cache's writer and reader on their own.
//
// All of it moves rows and does some ten operations per value, so memory is the bound.  A lane holds eight channels of one
// row (16 bytes of bf16), D / 8 lanes a row, so a wave has four rows of 128 channels (eight of 64): the same head of
// consecutive tokens, which in a block of the cache are one piece of 256 bytes of value codes.  Sums of squares, partners
// of the rotation and the largest magnitude of a group of 32 channels are then exchanges between lanes of a row, and the
// angles of a token stay in registers while a wave goes through the heads.
//
// Measured, where a copy of 2 GiB has 4.9 TB/s read and written: norms and rotation of 32768 tokens of 32 + 8 heads of 128 in
// bf16, 671 MB, 155-161 us, 4.2 TB/s (angles and weights of each token read again for every head: 435 us); 4001 tokens in
// fp32, 64 channels, 82 MB, 17-18 us; 16 tokens that are stored as well 5 us, a launch and three trips to memory.  419328 rows
// of 8 heads of 128 in bf16, 2.17 GB: 372 us to store (5.8 TB/s), 423 to load (5.1).
#include "kv4.hpp"

namespace shotkv {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kEnough = 2048;  // workgroups that fill the chip

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
template <typename T>
__device__ __forceinline__ void store8(char* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    __builtin_nontemporal_store(u32x4{to_bf16x2(x[0], x[1]), to_bf16x2(x[2], x[3]), to_bf16x2(x[4], x[5]), to_bf16x2(x[6], x[7])},
                                reinterpret_cast<u32x4*>(p));
  } else {
    __builtin_nontemporal_store(floatx4{x[0], x[1], x[2], x[3]}, reinterpret_cast<floatx4*>(p));
    __builtin_nontemporal_store(floatx4{x[4], x[5], x[6], x[7]}, reinterpret_cast<floatx4*>(p) + 1);
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

template <int D, typename T>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(RopeArgs a, int heads_per_group) {
  constexpr int kLanes = D / 8, kRows = kWave / kLanes;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int chunk = lane % kLanes, c0 = chunk * 8;
  const int t = (blockIdx.x * kWaves + wave) * kRows + lane / kLanes;
  const bool in_batch = t < a.T;
  const int tc = min(t, a.T - 1);
  const int pos = a.token_pos[tc];
  const bool live = in_batch && pos >= 0 && pos < a.n_positions;
  int slot = -1;
  if (a.cache.base && live) slot = a.slot_map[tc];
  const bool stored = static_cast<uint32_t>(slot) < a.cache.n_slots && a.cache.base;
  // cosine and signed sine of every channel: y = x * co + partner * si
  float co[8], si[8];
  const int half = a.rot_dim / 2;
  const float* row = a.table + static_cast<size_t>(live ? pos : 0) * a.rot_dim;
  const bool turns = c0 < a.rot_dim;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = c0 + i;
    const int pair = a.interleaved ? c >> 1 : c < half ? c : c - half;
    const bool second = a.interleaved ? c & 1 : c >= half;
    co[i] = turns ? row[pair] : 1.f;
    const float s = turns ? row[half + pair] : 0.f;
    si[i] = second ? s : -s;
  }
  // the lane that holds the other channels of this lane's pairs
  const int partner = !turns || a.interleaved ? lane : c0 < half ? lane + half / 8 : lane - half / 8;
  // this lane's place in the token's rows
  constexpr int kSize = sizeof(T);
  const char* const q_in = a.q.token(tc) + c0 * kSize;
  const char* const k_in = a.k.token(tc) + c0 * kSize;
  const char* const v_in = a.v.data ? a.v.token(tc) + c0 * kSize : nullptr;
  char* const q_out = a.q_out.token(tc) + c0 * kSize;
  char* const k_out = a.k_out.data ? a.k_out.token(tc) + c0 * kSize : nullptr;
  float q_weight[8], k_weight[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q_weight[i] = k_weight[i] = 1.f;
  if (a.q_weight) load8<T>(static_cast<const char*>(a.q_weight) + c0 * kSize, q_weight);
  if (a.k_weight) load8<T>(static_cast<const char*>(a.k_weight) + c0 * kSize, k_weight);
  const int all = a.H + a.H_kv + (a.cache.base ? a.H_kv : 0);  // query heads, key heads, value heads
  const int h_end = min(all, (static_cast<int>(blockIdx.y) + 1) * heads_per_group);
  auto row_of = [&](int h) {
    return h < a.H ? q_in + h * a.q.head_stride
                   : h < a.H + a.H_kv ? k_in + (h - a.H) * a.k.head_stride : v_in + (h - a.H - a.H_kv) * a.v.head_stride;
  };
  int h = blockIdx.y * heads_per_group;
  RawRow<T> next;
  if (h < h_end) next = fetch8<T>(row_of(h));
  for (; h < h_end; ++h) {
    float x[8];
    widen8<T>(next, x);
    if (h + 1 < h_end) next = fetch8<T>(row_of(h + 1));  // the next row, while this one is worked on
    const bool is_q = h < a.H;
    if (h >= a.H + a.H_kv) {
      put_row<D, true>(a.cache, slot, h - a.H - a.H_kv, chunk, stored, x);
      continue;
    }
    if (is_q ? a.q_weight : a.k_weight) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
      sum += __uint_as_float(lane_xor<1>(__float_as_uint(sum)));
      sum += __uint_as_float(lane_xor<2>(__float_as_uint(sum)));
      sum += __uint_as_float(lane_xor<4>(__float_as_uint(sum)));
      if (D == 128) sum += __uint_as_float(lane_xor<8>(__float_as_uint(sum)));
      const float inv = 1.f / sqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * (is_q ? q_weight[i] : k_weight[i]);
    }
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float other = a.interleaved ? x[i ^ 1] : __shfl(x[i], partner);
      y[i] = turns ? fmaf(x[i], co[i], other * si[i]) : x[i];
    }
    if (!live) {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = 0.f;
    }
    if (is_q) {
      if (in_batch) store8<T>(q_out + h * a.q_out.head_stride, y);
    } else {
      if (in_batch && k_out) store8<T>(k_out + (h - a.H) * a.k_out.head_stride, y);
      if (a.cache.base) {
        round8<T>(y);
        put_row<D, false>(a.cache, slot, h - a.H, chunk, stored, y);
      }
    }
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

}  // namespace

hipError_t launch_norm_rope(const RopeArgs& a, hipStream_t s) {
  const int tokens = kWave / (a.D / 8);  // of a wave
  // A wave keeps its tokens' angles through the heads that it goes through: all of them where that leaves enough
  // workgroups, fewer in short batches.  The four waves of a workgroup take neighbouring tokens, so that the rows that they
  // read and write together are 4 KB in a layout by head (32768 tokens of 32 + 8 heads of 128 in 158 us; with a head each
  // of the same four tokens 177).
  const int all = a.H + a.H_kv + (a.cache.base ? a.H_kv : 0);
  const int quads = ceil_div(a.T, tokens * kWaves);
  const int groups = min(ceil_div(kEnough, quads), all);
  const int per_group = ceil_div(all, groups);
  const dim3 grid(quads, ceil_div(all, per_group));
  if (a.D == 128) {
    if (a.dtype == SHOTKV_BF16) norm_rope_kernel<128, bf16_t><<<grid, kThreads, 0, s>>>(a, per_group);
    else norm_rope_kernel<128, float><<<grid, kThreads, 0, s>>>(a, per_group);
  } else {
    if (a.dtype == SHOTKV_BF16) norm_rope_kernel<64, bf16_t><<<grid, kThreads, 0, s>>>(a, per_group);
    else norm_rope_kernel<64, float><<<grid, kThreads, 0, s>>>(a, per_group);
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
