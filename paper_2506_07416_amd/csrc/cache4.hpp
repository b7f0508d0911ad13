// Layout of the 4-bit cache and the decoding of its codes (gfx950).
#pragma once

#include "common.hpp"

namespace litevlm {

constexpr int kCacheBlock = 32;  // elements that share one E8M0 scale

// The four arrays of one (sample, KV head); offsets in bytes fit 32 bits for
// cap <= LITEVLM_MAX_CACHE4 (2^24 * 136 < 2^32).
template <int D>
struct CacheHead {
  static constexpr uint32_t kRow = D / 2;             // code bytes of a row
  static constexpr uint32_t kBlocks = D / kCacheBlock;
  uint8_t* kc;
  uint8_t* vc;
  uint8_t* ks;
  uint8_t* vs;
  __host__ __device__ static int64_t bytes(int cap) { return (int64_t)cap * (D + D / 16); }
  __device__ __forceinline__ CacheHead(const uint8_t* cache, int64_t head, int cap) {
    kc = const_cast<uint8_t*>(cache) + head * bytes(cap);
    vc = kc + (int64_t)cap * kRow;
    ks = vc + (int64_t)cap * kRow;
    vs = ks + (int64_t)cap * kBlocks;
  }
};

// The conversions take an E8M0 scale from the exponent bits of a float; exponent
// 255 gives NaN, exponent 0 is 2^-127 (all as E8M0 has it).
__device__ __forceinline__ float e8m0_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight E2M1 codes of one block (element 0 in the low bits) to bf16, exactly.
__device__ __forceinline__ bf16x8 decode8(uint32_t w, float scale) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const auto d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The two codes of byte j (a constant after unrolling) of w, as packed bf16.
__device__ __forceinline__ uint32_t decode2(uint32_t w, float scale, int j) {
  return __builtin_bit_cast(uint32_t, j == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)
                                      : j == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)
                                      : j == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)
                                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
}

}  // namespace litevlm
