// Rows of queries, keys and values on their way to attention: per-head norms and rotation in one pass, with the keys and
// values of new tokens going straight into the 4-bit cache, and the cache's writer and reader on their own.
//
// All of it moves rows and does some ten operations per value, so memory is the bound.  A lane holds eight channels of one
// row (16 bytes of bf16), D / 8 lanes a row, so a wave has four rows of 128 channels (eight of 64): the same head of
// consecutive tokens, which in a block of the cache are one piece of 256 bytes of value codes.  Sums of squares, partners
// of the rotation and the largest magnitude of a group of 32 channels are then exchanges between lanes of a row, and the
// angles of a token stay in registers while a wave goes through the heads.
#include "kv4.hpp"

namespace shotkv {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

template <typename T>
__device__ __forceinline__ void load8(const char* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const u32x4 raw = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(raw[i] << 16);
      x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
    }
  } else {
    const u32x4 a = reinterpret_cast<const u32x4*>(p)[0], b = reinterpret_cast<const u32x4*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = __uint_as_float(a[i]);
      x[4 + i] = __uint_as_float(b[i]);
    }
  }
}
typedef __attribute__((ext_vector_type(2))) float floatx2;
__device__ __forceinline__ uint32_t to_bf16x2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{a, b}), bf16x2));
}
template <typename T>
__device__ __forceinline__ void store8(char* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x4*>(p) = u32x4{to_bf16x2(x[0], x[1]), to_bf16x2(x[2], x[3]), to_bf16x2(x[4], x[5]), to_bf16x2(x[6], x[7])};
  } else {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
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
  const int t = blockIdx.x * kRows + lane / kLanes;
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
  const int all = a.H + a.H_kv + (a.cache.base ? a.H_kv : 0);
  const int h_end = min(all, (static_cast<int>(blockIdx.y) + 1) * heads_per_group);
  for (int h = blockIdx.y * heads_per_group + wave; h < h_end; h += kWaves) {
    const bool is_q = h < a.H, is_v = h >= a.H + a.H_kv;
    const int hh = is_q ? h : is_v ? h - a.H - a.H_kv : h - a.H;
    const RowView& in = is_q ? a.q : is_v ? a.v : a.k;
    float x[8];
    load8<T>(in.token(tc) + hh * in.head_stride + c0 * sizeof(T), x);
    if (is_v) {
      put_row<D, true>(a.cache, slot, hh, chunk, stored, x);
      continue;
    }
    const void* weight = is_q ? a.q_weight : a.k_weight;
    if (weight) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
      sum += __uint_as_float(lane_xor<1>(__float_as_uint(sum)));
      sum += __uint_as_float(lane_xor<2>(__float_as_uint(sum)));
      sum += __uint_as_float(lane_xor<4>(__float_as_uint(sum)));
      if (D == 128) sum += __uint_as_float(lane_xor<8>(__float_as_uint(sum)));
      const float inv = 1.f / sqrtf(sum * (1.f / D) + a.eps);
      float w[8];
      load8<T>(static_cast<const char*>(weight) + c0 * sizeof(T), w);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * w[i];
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
    const RowView& out = is_q ? a.q_out : a.k_out;
    if (in_batch && out.data) store8<T>(out.token(t) + hh * out.head_stride + c0 * sizeof(T), y);
    if (!is_q && a.cache.base) {
      round8<T>(y);
      put_row<D, false>(a.cache, slot, hh, chunk, stored, y);
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
      load8<T>(k + h * a.k.head_stride, x);
      load8<T>(v + h * a.v.head_stride, y);
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
  const int all = a.H + a.H_kv + (a.cache.base ? a.H_kv : 0);
  const int groups = ceil_div(all, kWaves);
  const dim3 grid(ceil_div(a.T, tokens), groups);
  if (a.D == 128) {
    if (a.dtype == SHOTKV_BF16) norm_rope_kernel<128, bf16_t><<<grid, kThreads, 0, s>>>(a, kWaves);
    else norm_rope_kernel<128, float><<<grid, kThreads, 0, s>>>(a, kWaves);
  } else {
    if (a.dtype == SHOTKV_BF16) norm_rope_kernel<64, bf16_t><<<grid, kThreads, 0, s>>>(a, kWaves);
    else norm_rope_kernel<64, float><<<grid, kThreads, 0, s>>>(a, kWaves);
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
