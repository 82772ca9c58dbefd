// The paged 4-bit cache: layout, coding of rows and launchers.
#pragma once

#include "common.hpp"

namespace shotkv {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kKv4Block = 32;       // tokens of a block
constexpr uint32_t kKv4NotFinite = 255;

// Where things are in a block of 32 tokens of one KV head (34 * D bytes).
template <int D>
struct Kv4Block {
  static constexpr int kKeys = 0;                  // [32][D / 2]
  static constexpr int kValues = 16 * D;           // [8 quads][D / 8][4 tokens][4 bytes]
  static constexpr int kKeyScales = 32 * D;        // [32][D / 32]
  static constexpr int kValueScales = 33 * D;      // [8 quads][D / 32][4 tokens]
  static constexpr int kBytes = 34 * D;
  static __device__ __forceinline__ int key_word(int token, int chunk) { return kKeys + token * (D / 2) + chunk * 4; }
  static __device__ __forceinline__ int value_word(int token, int chunk) {
    return kValues + ((token >> 2) * (D / 8) + chunk) * 16 + (token & 3) * 4;
  }
  static __device__ __forceinline__ int key_scale(int token, int group) { return kKeyScales + token * (D / 32) + group; }
  static __device__ __forceinline__ int value_scale(int token, int group) {
    return kValueScales + ((token >> 2) * (D / 32) + group) * 4 + (token & 3);
  }
};

inline size_t kv4_page_bytes(int page_size, int H_kv, int D) { return static_cast<size_t>(H_kv) * page_size / 32 * 34 * D; }

// Device view of a cache.
struct Kv4Pages {
  char* base;
  uint32_t n_slots;    // n_pages * page_size
  int n_pages;
  int page_shift;      // log2(page_size)
  int H_kv;
};

// Block and token of a slot: byte offset of the block that holds it for one KV head.
template <int D>
__device__ __forceinline__ size_t kv4_block_offset(const Kv4Pages& c, uint32_t page, int head, uint32_t block_in_page) {
  return ((static_cast<size_t>(page) * c.H_kv + head) * (1u << (c.page_shift - 5)) + block_in_page) * Kv4Block<D>::kBytes;
}
template <int D>
__device__ __forceinline__ char* kv4_block_of_slot(const Kv4Pages& c, uint32_t slot, int head) {
  const uint32_t in_page = slot & ((1u << c.page_shift) - 1u);
  return c.base + kv4_block_offset<D>(c, slot >> c.page_shift, head, in_page >> 5);
}

// Eight values of a lane as one word of codes, and the scale byte of the group of 32 channels that four lanes hold.
// The scale is the least power of two whose seven-fold is no less than the largest magnitude: magnitudes between 6 and 7
// round to 6, no further off than anything between 4 and 6 may be.  On the bits of the largest magnitude: its exponent
// less 2, one more where the mantissa is over 1.75.  The comparison is of bits, so that a NaN counts as the largest.
__device__ __forceinline__ uint32_t kv4_encode(const float (&x)[8], uint32_t* scale_byte) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
  most = max(most, lane_xor<1>(most));
  most = max(most, lane_xor<2>(most));
  int e = static_cast<int>((most + 0x1fffffu) >> 23) - 2;
  e = min(max(e, 1), 252);
  const bool finite = most < 0x7f800000u;
  const float scale = __uint_as_float(static_cast<uint32_t>(e) << 23);
  uint32_t codes = 0;  // the conversion divides by the scale, rounds to nearest even and holds at 6
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
  *scale_byte = finite ? static_cast<uint32_t>(e) : kKv4NotFinite;
  return finite ? codes : 0u;
}

// The scale that a byte stands for, as the conversions below take it (by the exponent of a float: 255 gives NaN).
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

__device__ __forceinline__ void kv4_decode(uint32_t codes, float scale, float (&x)[8]) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1),
              c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1]; x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
}

// Rows of D elements anywhere (shotkv_rows), as the kernels take them: strides in bytes.
struct RowView {
  char* data;
  long long seq_stride, token_stride, head_stride;
  int seq_tokens;
  __device__ __forceinline__ char* token(int t) const {
    const int s = t / seq_tokens;
    return data + s * seq_stride + (t - s * seq_tokens) * token_stride;
  }
};

// ---- launchers -----------------------------------------------------------------------------------

hipError_t launch_pages_plan(int R, int page_shift, int max_pages, const int32_t* cached_lens, const int32_t* new_lens,
                             const int32_t* pos_start, const int32_t* free_pages, int stack_size,
                             const int32_t* free_count, int32_t* block_table, int32_t* free_left, int32_t* seq_lens,
                             int32_t* query_start, int T, int request_tokens, int32_t* slot_map, int32_t* token_pos,
                             int32_t* status, hipStream_t s);
hipError_t launch_pages_release(int R, int page_shift, int max_pages, const uint8_t* finished, int32_t* seq_lens,
                                int32_t* block_table, int32_t* free_pages, int stack_size, int32_t* free_count,
                                hipStream_t s);

struct RopeArgs {
  int T, H, H_kv, D, dtype;
  const float* table;
  int n_positions, rot_dim, interleaved;
  float eps;
  const void *q_weight, *k_weight;
  const int32_t* token_pos;
  RowView q, k, v, q_out, k_out;  // v.data and k_out.data may be null
  Kv4Pages cache;                 // base may be null
  const int32_t* slot_map;
};
hipError_t launch_norm_rope(const RopeArgs& a, hipStream_t s);

struct Kv4RowArgs {
  int T, D, dtype;
  RowView k, v;
  Kv4Pages cache;
  const int32_t* slot_map;
};
hipError_t launch_kv4_store(const Kv4RowArgs& a, hipStream_t s);
hipError_t launch_kv4_load(const Kv4RowArgs& a, hipStream_t s);

struct Kv4AttentionArgs {
  int R, T, H, H_kv, G, D, dtype, max_q_len, max_pages;
  float sm_scale;
  Kv4Pages cache;
  const int32_t *block_table, *seq_lens, *query_start;
  RowView q, out;
  float* lse;
};

}  // namespace shotkv
