// Elements of the cache's and the activations' types, shared by the kernels that deal with values
// (vtoken_rows.hip, vtoken_prompt.hip). Not installed.
#pragma once

#include <type_traits>

#include "vtoken_internal.h"

namespace vtoken {
namespace elements {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
// the same in a caller's float buffers, which are aligned to a float and no more
typedef f32x2 f32x2_in __attribute__((aligned(4)));
typedef f32x4 f32x4_in __attribute__((aligned(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));

// The 16-bit type of activations and of matrix-core operands. Softmax weights are 2^(x - m): m follows
// a row's maximum, to kFirst below it, where that passes m + kMost, so that the sums so far are seldom
// scaled. A row's largest weight then lies between 2^kFirst and 2^kMost. fp16 ends at 2^-24: from 2^11
// on, a weight is off by 2^-36 of the largest at most where fp16's relative steps end (from 1 on it was
// 2^-25, and tens of thousands of keys far below the largest were lost).
template <bool kBf16>
struct Act {
  static constexpr float kFirst = 11.f, kMost = 15.f;
  typedef _Float16 elem;
  typedef f16x8 x8;
  typedef f16x2 x2;
};
template <>
struct Act<true> {
  static constexpr float kFirst = 0.f, kMost = 8.f;
  typedef __bf16 elem;
  typedef bf16x8 x8;
  typedef bf16x2 x2;
};

// e8m0 exponent -> 2^(e - 127) (255: NaN, 0: zero, which no stored row has).
__device__ __forceinline__ float e8m0_scale(uint32_t e) {
  return e == 255 ? __builtin_nanf("") : __uint_as_float(e << 23);
}

// Eight consecutive elements of a cache row as activations: 16 bytes of fp16 / bf16 as they are,
// 8 bytes of fp8 or 4 bytes of codes through the conversion instructions. Every value is exact
// (e4m3 in fp16 and bf16, e2m1 times a power of two in bf16).
template <bool kBf16>
__device__ __forceinline__ u32x4 widen_fp8(u32x2 w) {
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (kBf16) {
      o[2 * i] = __builtin_bit_cast(
          uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(w[i]), 1.f, false));
      o[2 * i + 1] = __builtin_bit_cast(
          uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(w[i]), 1.f, true));
    } else {
      o[2 * i] = __builtin_bit_cast(
          uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(w[i]), 1.f, false));
      o[2 * i + 1] = __builtin_bit_cast(
          uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(w[i]), 1.f, true));
    }
  }
  return o;
}

__device__ __forceinline__ u32x4 widen_fp4(uint32_t w, float scale) {
  u32x4 o;
  o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return o;
}

// LDS addresses, 32 bits wide.
typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
typedef __attribute__((address_space(3))) uint32_t lds_u32;
typedef __attribute__((address_space(3))) uint16_t lds_u16;

// Rows of 16-bit values lie in LDS without padding (loads that write it directly leave none), 16-byte
// piece c of row r at c ^ swizzle(r): the 16-byte reads of 16 rows at one c, and transpose reads of
// 4 rows x 64 bytes or 8 rows x 32 bytes, then fall on different banks.
template <int kD>
__device__ __forceinline__ int swizzle(int r) {
  const int low = (r >> 1 & 2) | (r >> 3 & 1);
  return kD >= 128 ? (r & 3) << 2 | low : kD == 64 ? (r >> 1 & 1) << 2 | low : low;
}
template <int kD>
__device__ __forceinline__ int piece_at(int r, int c) {   // byte offset
  return r * (kD * 2) + ((c ^ swizzle<kD>(r)) << 4);
}

// A lane's 16 loaded bytes of fp8 or codes become 2 or 4 pieces of such a row. Written in order the
// pieces of 16 neighbouring lanes would meet on the same banks: lane `ln` of row r writes piece
// y ^ write_turn(r, ln) y-th.
template <int kKind, int kD>
__device__ __forceinline__ int write_turn(int r, int ln) {
  if constexpr (kKind == 3) {
    return kD == 256 ? (ln >> 2 & 1) | (r & 1) << 1 : kD == 128 ? r & 3 : kD == 64 ? r >> 1 & 1 : 0;
  } else {
    return kD == 256 ? ln >> 3 & 1 : kD == 128 ? r & 1 : kD == 64 ? r >> 1 & 1 : r >> 2 & 1;
  }
}

// The pieces of 16 bytes of a cache row in the order in which they are written.
template <bool kBf16, int kKind>
__device__ __forceinline__ void widen(u32x4 w, float scale, int turn, u32x4* o) {
  if constexpr (kKind == 3) {
    const bool one = (turn & 1) != 0, two = (turn & 2) != 0;
    const u32x4 x = {one ? w.y : w.x, one ? w.x : w.y, one ? w.w : w.z, one ? w.z : w.w};
    o[0] = widen_fp4(two ? x.z : x.x, scale);
    o[1] = widen_fp4(two ? x.w : x.y, scale);
    o[2] = widen_fp4(two ? x.x : x.z, scale);
    o[3] = widen_fp4(two ? x.y : x.w, scale);
  } else {
    const bool one = turn != 0;
    o[0] = widen_fp8<kBf16>(one ? u32x2{w.z, w.w} : u32x2{w.x, w.y});
    o[1] = widen_fp8<kBf16>(one ? u32x2{w.x, w.y} : u32x2{w.z, w.w});
  }
}

// LDS transpose read (ds_read_b64_tr_b16): in each group of 16 lanes, lane 4a + b receives element
// b of the four 16-bit values addressed by lanes a, a+4, a+8 and a+12 of its group.
__device__ __forceinline__ i16x4 lds_read_tr16(const lds_u8* at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)at);
}

}  // namespace elements
}  // namespace vtoken
