// Blocks of the paged 4-bit cache on their way to a wave, for the attention kernels whose waves take blocks by themselves.
#pragma once

#include "kv4_attention.hpp"

namespace shotkv {

// Blocks on their way: every wave has a ring of them in LDS that it fills and reads by itself, straight from memory
// (global_load_lds: lane l's 16 bytes go to 16 l), so what is in flight takes no registers and waits for nobody.  Keys of 128
// channels are fetched so that lane l finds its codes at 16 l as well.
template <int D, int DEPTH>
struct Ring {
  static constexpr int kSlot = 32 * D + 256;  // codes, and the scales (of 128 bytes in D = 64, twice)
  static constexpr int kDepth = DEPTH;
  static constexpr int kBytes = kDepth * kSlot;  // of a wave
};

// The slot has the block's own layout (an instruction's offset counts in memory and in LDS).
template <int D>
__device__ __forceinline__ void request_block(const char* base, uint32_t slot, uint32_t key_piece, uint32_t straight, uint32_t word) {
  typedef Kv4Block<D> B;
  if constexpr (D == 128) {
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %2, %5 nt\n\tglobal_load_lds_dwordx4 %2, %5 offset:%6 nt\n\t"
        "global_load_lds_dwordx4 %3, %5 offset:%7 nt\n\tglobal_load_lds_dwordx4 %3, %5 offset:%8 nt\n\t"
        "s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %4, %5 nt"
        :
        : "s"(slot), "s"(slot + B::kKeyScales), "v"(key_piece), "v"(straight), "v"(word), "s"(base), "n"(kWave * 16), "n"(B::kValues),
          "n"(B::kValues + kWave * 16)
        : "memory", "m0");
  } else {
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %3 nt\n\tglobal_load_lds_dwordx4 %1, %3 offset:%4 nt\n\t"
        "global_load_lds_dword %2, %3 offset:%5 nt"
        :
        : "s"(slot), "v"(straight), "v"(word), "s"(base), "n"(B::kValues), "n"(B::kKeyScales)
        : "memory", "m0");
  }
}
// The oldest block has arrived; one younger may still be on its way.
template <int D, int DEPTH>
__device__ __forceinline__ void wait_block(bool younger) {
  static_assert(DEPTH == 2, "one block besides the oldest");
  constexpr int kLoads = D == 128 ? 5 : 3;  // instructions of a block
  if (younger) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kLoads) : "memory");
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

}  // namespace shotkv
