// The 8-bit cache's codes four at a time, and what its two writes share.
#pragma once

#include <stdint.h>

#include "f32x2.cuh"
#include "serve.cuh"

namespace seedq {

// Four codes of the products x times a number, where none is past the largest code.
// int8: 1.5 * 2^23 has unit 1, so adding it rounds to an integer in the low bits.
template <int KIND>
__device__ __forceinline__ uint32_t four_codes(uint64_t x01, uint64_t x23, uint64_t by2) {
  if (KIND == SEEDQ_KV_INT8) {
    const uint64_t one = f2_pack(12582912.f, 12582912.f);
    const float2 a = f2_unpack(f2_add(f2_mul(x01, by2), one)), b = f2_unpack(f2_add(f2_mul(x23, by2), one));
    return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040),
                       __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
  }
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(f2_unpack(f2_mul(x01, by2)), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(f2_unpack(f2_mul(x23, by2)), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}
// The numbers of four codes, in pairs.  int8: byte + 128 in the low bits of 2^23.
template <int KIND>
__device__ __forceinline__ void four_values(uint32_t w, uint64_t &x01, uint64_t &x23) {
  if (KIND == SEEDQ_KV_INT8) {
    const uint32_t y = w ^ 0x80808080u;
    const uint64_t off = f2_pack(-8388736.f, -8388736.f);
    auto wide = [&](int sel) { return __uint_as_float(__byte_perm(y, 0x4b000000u, sel)); };
    x01 = f2_add(f2_pack(wide(0x7440), wide(0x7441)), off);
    x23 = f2_add(f2_pack(wide(0x7442), wide(0x7443)), off);
  } else {
    const uint32_t lo = e4m3x2_to_half2(w), hi = e4m3x2_to_half2(w >> 16);
    const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&lo));
    const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
    x01 = f2_pack(a.x, a.y), x23 = f2_pack(b.x, b.y);
  }
}

// log2 of the tokens whose stretches on a page a warp of the append owns.
inline int32_t append_group_shift(int64_t tokens, int32_t heads) {
  // One token per warp until the warps fill the GPU twice over, then more.  Each may
  // be a page of its own (32 heads, 256 single tokens: 10.4 us, with one token per
  // warp 11.5, with 32 38; 512: 17, 21 and 40), or all on a page (4 prompts of 1024,
  // pages of 64: 23 us, with one token per warp 77, with 32 24).  At half the
  // threshold 256 single tokens take 9.5 and the prompts as long, at twice 11.6 and 28.
  int32_t shift = 0;
  while (shift < 5 && (tokens >> shift) * heads * 2 > 2 * 152 * 48) ++shift;
  return shift;
}

}  // namespace seedq
