// Rows of the cache as values (vtoken_write_kv, vtoken_read_kv).
//
//   write_kernel   per-head RMS norm and rotation of q and k, k and v stored at their slots in the
//                  cache's type, q to its output
//   read_kernel    rows of listed slots widened to dense 16-bit tensors
//
// A head row is taken by a group of lanes, eight elements (16 bytes) each, so that a group reads
// its row with one load per lane, reduces and turns it in registers and stores it: every byte is
// moved once. A group takes kRowsPer rows of a token one after the other: their loads are in flight
// together, and the angles, the weights and the token's slot and position are read once for them.
// Large calls move at the rate of a library's copy of 4 GiB (4.7 TB/s), which is not the memory's: probes
// on this card read at 7.2 TB/s, write at 6.1 and copy at 6.2. Small ones are bound by latency. 8,192 tokens
// of 32 query and 8 KV heads of 128 into a 16-bit cache (206 MB, half of them written) take 44 us, 4.6 TB/s,
// where those rates give 31; 4,097 tokens of 64 query heads into a 4-bit cache (158 MB) 38 us, 4.1 TB/s;
// 65,536 tokens' 4-bit rows read (340 MB, four fifths written) 66 us, 5.1 TB/s, where the rates give 54; one
// token 4 us. With one head row to a group the first took 70 us and the last but one 96; with four of mixed
// kinds the first took 54.
#include "vtoken_elements.h"

namespace vtoken {
namespace {

using namespace elements;

constexpr int kRowThreads = 256;
constexpr int kRowsPer = 4;

// The value of another lane of the 16-lane row (DPP control word), without LDS.
template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, 0xF, 0xF, false));
}
// Exchange with lane i ^ 1, i ^ 2, 3 - i of a quad, 7 - i of eight, 15 - i and (i + 8) % 16 of a row.
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kQuadMirror = 0x1B, kHalfMirror = 0x141, kMirror = 0x140,
              kRor8 = 0x128;

template <int kCtrl>
__device__ __forceinline__ double dpp_add(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint64_t v = static_cast<uint64_t>(dpp<kCtrl>(static_cast<uint32_t>(u >> 32))) << 32 |
                     dpp<kCtrl>(static_cast<uint32_t>(u));
  return x + __builtin_bit_cast(double, v);
}

// Sum over a group of kLanes lanes (all of them active).
template <int kLanes>
__device__ __forceinline__ double group_sum(double x) {
  x = dpp_add<kXor1>(x);
  x = dpp_add<kXor2>(x);
  if constexpr (kLanes >= 8) x = dpp_add<kHalfMirror>(x);
  if constexpr (kLanes >= 16) x = dpp_add<kMirror>(x);
  if constexpr (kLanes == 32) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = static_cast<uint32_t>(u), hi = static_cast<uint32_t>(u >> 32);
    const auto l = __builtin_amdgcn_permlane16_swap(lo, lo, false, false);
    const auto h = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    x = __builtin_bit_cast(double, static_cast<uint64_t>(h[0]) << 32 | l[0]) +
        __builtin_bit_cast(double, static_cast<uint64_t>(h[1]) << 32 | l[1]);
  }
  return x;
}

// The value of the lane half a group on.
template <int kLanes>
__device__ __forceinline__ float other_half(float x) {
  const uint32_t u = __float_as_uint(x);
  if constexpr (kLanes == 4) return __uint_as_float(dpp<kXor2>(u));
  if constexpr (kLanes == 8) return __uint_as_float(dpp<kQuadMirror>(dpp<kHalfMirror>(u)));
  if constexpr (kLanes == 16) return __uint_as_float(dpp<kRor8>(u));
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 16) != 0 ? r[0] : r[1]);
}

// 1 / sqrt(v) to the last bits of a double (two Newton steps from the instruction's estimate; a
// quarter of the time of a root and a division).
__device__ __forceinline__ double inverse_root(double v) {
  double y = __builtin_amdgcn_rsq(v);
  if (y == 0.) return y;   // of an infinity
#pragma unroll
  for (int i = 0; i < 2; ++i) y = fma(0.5 * y, fma(-v * y, y, 1.), y);
  return y;
}

template <bool kBf16>
__device__ __forceinline__ void to_float(u32x4 w, float (&x)[8]) {
  const auto e = __builtin_bit_cast(typename Act<kBf16>::x8, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(e[i]);
}

template <bool kBf16>
__device__ __forceinline__ u32x4 to_act(const float (&x)[8]) {
  typename Act<kBf16>::x8 e;
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = static_cast<typename Act<kBf16>::elem>(x[i]);
  return __builtin_bit_cast(u32x4, e);
}

// Stores a lane's eight values of head h (lane `sub` of its group) into a cache row.
template <bool kBf16, int kKind>
__device__ __forceinline__ void store_row(uint8_t* row, int heads, int head_dim, int h, int sub,
                                          const float (&x)[8]) {
  if constexpr (kKind <= 1) {
    *reinterpret_cast<u32x4*>(row + (h * head_dim + sub * 8) * 2) = to_act<kBf16>(x);
  } else if constexpr (kKind == 2) {
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {   // saturates, keeps NaN
        const float y = x[4 * i + j];
        c[j] = y != y ? y : fminf(fmaxf(y, -448.f), 448.f);
      }
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
      p = __builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], p, true);
      w[i] = static_cast<uint32_t>(p);
    }
    *reinterpret_cast<u32x2*>(row + h * head_dim + sub * 8) = w;
  } else {
    // the exponent of the four lanes' 32 values: bits compare as their magnitudes do, NaN highest
    int top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_int(x[i]) & 0x7fffffff);
    top = max(top, static_cast<int>(dpp<kXor1>(top)));
    top = max(top, static_cast<int>(dpp<kXor2>(top)));
    const int field = top >> 23;
    const int e = field == 255 ? 255 : max(field - 2, 1);
    // x / 2^(e - 127) to the nearest code, ties to even ones, 6 at most
    const float scale = __int_as_float(min(e, 254) << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    if (e == 255) w = 0;
    *reinterpret_cast<uint32_t*>(row + h * (head_dim / 2) + sub * 4) = w;
    if ((sub & 3) == 0) {
      row[heads * (head_dim / 2) + h * (head_dim / 32) + sub / 4] = static_cast<uint8_t>(e);
    }
  }
}

// Eight floats of a caller's buffer.
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4_in*>(p);
  const f32x4 b = *reinterpret_cast<const f32x4_in*>(p + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = a[j];
    x[4 + j] = b[j];
  }
}

// kLanes: lanes per head row (the power of two from head_dim / 8 on, at least 4). A group's rows are
// all queries, all keys or all values.
template <int kLanes, bool kBf16, int kKind>
__global__ __launch_bounds__(kRowThreads) void write_kernel(WriteArgs a) {
  // the results decide roundings to 8 and 4 bits: no contraction, the formula's own roundings
#pragma clang fp contract(off)
  const int D = a.head_dim;
  const uint32_t q_parts = (a.num_q_heads + kRowsPer - 1) / kRowsPer;
  const uint32_t kv_parts = (a.num_kv_heads + kRowsPer - 1) / kRowsPer;
  const uint32_t parts = q_parts + 2 * kv_parts;
  const uint32_t group = (blockIdx.x * kRowThreads + threadIdx.x) / kLanes;
  const uint32_t tok = group / parts;
  if (tok >= static_cast<uint32_t>(a.num_tokens)) return;   // (whole groups: they exchange values)
  const uint32_t part = group - tok * parts;
  const bool is_q = part < q_parts, is_v = part >= q_parts + kv_parts;
  const uint32_t in_kind = part - (is_q ? 0u : is_v ? q_parts + kv_parts : q_parts);
  const int h0 = static_cast<int>(in_kind) * kRowsPer;
  const int n = min(kRowsPer, (is_q ? a.num_q_heads : a.num_kv_heads) - h0);   // rows of the group
  const int64_t t = tok;
  const int slot = a.slots[t];
  const int sub = threadIdx.x % kLanes;
  const int e = sub * 8;
  const bool full = D == kLanes * 8;      // (uniform) no lane is past the row
  const bool mine = full || e < D;

  const uint8_t* src = (is_q ? a.q : is_v ? a.v : a.k) +
                       (t * (is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride) +
                        (int64_t)h0 * D + (mine ? e : 0)) * 2;
  u32x4 raw[kRowsPer];
#pragma unroll
  for (int j = 0; j < kRowsPer; ++j) {
    raw[j] = *reinterpret_cast<const u32x4*>(src + min(j, n - 1) * (D * 2));
  }
  if (slot < 0) return;
  const int half = a.rotary_dim / 2;
  int pos = 0;
  if (half > 0) pos = a.positions[t];
  const bool bad =
      slot >= a.num_slots ||
      (half > 0 && static_cast<uint32_t>(pos) >= static_cast<uint32_t>(a.num_positions));
  uint8_t* row = (is_v ? a.vplane : a.kplane) + (bad ? 0 : slot) * a.row_bytes;
  if (is_v) {
    if (bad || !mine) return;
#pragma unroll
    for (int j = 0; j < kRowsPer; ++j) {
      if (j >= n) break;
      if constexpr (kKind <= 1) {
        *reinterpret_cast<u32x4*>(row + ((h0 + j) * D + e) * 2) = raw[j];
      } else {
        float x[8];
        to_float<kBf16>(raw[j], x);
        store_row<kBf16, kKind>(row, a.num_kv_heads, D, h0 + j, sub, x);
      }
    }
    return;
  }

  // the angles of this lane's values: pairs (2 j, 2 j + 1), or values at and half / 8 lanes on
  const bool turns = e < a.rotary_dim;
  float c[8] = {}, s[8] = {};
  if (turns) {
    const float* cs = a.cos_sin + (bad ? 0 : (int64_t)pos * a.rotary_dim);
    if (a.interleaved) {
      const f32x4 x = *reinterpret_cast<const f32x4_in*>(cs + e / 2);
      const f32x4 y = *reinterpret_cast<const f32x4_in*>(cs + half + e / 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c[j] = x[j];
        s[j] = y[j];
      }
    } else {
      const int at = e < half ? e : e - half;
      load8(cs + at, c);
      load8(cs + half + at, s);
    }
    // (a, b) -> (a c - b s, b c + a s): the first half's sines with their sign changed
    if (!a.interleaved && e < half) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = -s[j];
    }
  }
  const float* w = is_q ? a.q_weight : a.k_weight;
  float weight[8] = {};
  if (w != nullptr && mine) load8(w + e, weight);
  if (bad) {   // (queries: NaN; nothing of keys is stored)
#pragma unroll
    for (int j = 0; j < kRowsPer; ++j) raw[j] = u32x4{0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu};
  }
  uint8_t* out = is_q ? a.q_out + (t * a.q_out_stride + (int64_t)h0 * D + e) * 2 : nullptr;
#pragma unroll
  for (int j = 0; j < kRowsPer; ++j) {
    float x[8];
    to_float<kBf16>(raw[j], x);
    if (w != nullptr) {
      double sum = 0.;
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const double z = x[y];
        sum = fma(z, z, sum);
      }
      if (!mine) sum = 0.;
      const float r =
          static_cast<float>(inverse_root(group_sum<kLanes>(sum) * a.inv_dim + a.eps));
#pragma unroll
      for (int y = 0; y < 8; ++y) x[y] = x[y] * r * weight[y];
    }
    if (half > 0) {
      if (a.interleaved) {
        if (turns) {
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float p = x[2 * y], q = x[2 * y + 1];
            x[2 * y] = p * c[y] - q * s[y];
            x[2 * y + 1] = q * c[y] + p * s[y];
          }
        }
      } else if (a.rotary_dim == kLanes * 8) {
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const float o = other_half<kLanes>(x[y]);
          x[y] = x[y] * c[y] + o * s[y];
        }
      } else {
        const int from = (threadIdx.x & 63) + (e < half ? half / 8 : -(half / 8));
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const float o = __shfl(x[y], from & 63, 64);
          const float z = x[y] * c[y] + o * s[y];
          x[y] = turns ? z : x[y];
        }
      }
    }
    if (j >= n || !mine) continue;
    if (is_q) {
      *reinterpret_cast<u32x4*>(out + j * (D * 2)) = to_act<kBf16>(x);
    } else if (!bad) {
      store_row<kBf16, kKind>(row, a.num_kv_heads, D, h0 + j, sub, x);
    }
  }
}

// A lane's eight values of head h from a cache row, as activations.
template <bool kBf16, int kKind>
__device__ __forceinline__ u32x4 load_row(const uint8_t* row, int heads, int head_dim, int h,
                                          int sub) {
  if constexpr (kKind <= 1) {
    return *reinterpret_cast<const u32x4*>(row + (h * head_dim + sub * 8) * 2);
  } else if constexpr (kKind == 2) {
    return widen_fp8<kBf16>(*reinterpret_cast<const u32x2*>(row + h * head_dim + sub * 8));
  } else {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(row + h * (head_dim / 2) + sub * 4);
    return widen_fp4(
        w, e8m0_scale(row[heads * (head_dim / 2) + h * (head_dim / 32) + sub / 4]));
  }
}

template <int kLanes, bool kBf16, int kKind>
__global__ __launch_bounds__(kRowThreads) void read_kernel(ReadArgs a) {
  const uint32_t kv_parts = (a.num_kv_heads + kRowsPer - 1) / kRowsPer;
  const uint32_t group = (blockIdx.x * kRowThreads + threadIdx.x) / kLanes;
  const int sub = threadIdx.x % kLanes;
  const uint32_t tok = group / (2 * kv_parts);
  if (tok >= static_cast<uint32_t>(a.num_tokens) || sub * 8 >= a.head_dim) return;
  const uint32_t part = group - tok * 2 * kv_parts;
  const bool is_v = part >= kv_parts;
  const int h0 = static_cast<int>(is_v ? part - kv_parts : part) * kRowsPer;
  const int n = min(kRowsPer, a.num_kv_heads - h0);
  const int64_t t = tok;
  const int slot = a.slots[t];
  const bool ok = static_cast<unsigned>(slot) < static_cast<unsigned>(a.num_slots);
  const uint8_t* row = (is_v ? a.vplane : a.kplane) + (ok ? slot : 0) * a.row_bytes;
  u32x4 w[kRowsPer];
#pragma unroll
  for (int j = 0; j < kRowsPer; ++j) {
    w[j] = load_row<kBf16, kKind>(row, a.num_kv_heads, a.head_dim, h0 + min(j, n - 1), sub);
  }
  uint8_t* out = (is_v ? a.v_out + t * a.v_stride * 2 : a.k_out + t * a.k_stride * 2) +
                 ((int64_t)h0 * a.head_dim + sub * 8) * 2;
#pragma unroll
  for (int j = 0; j < kRowsPer; ++j) {
    if (j >= n) break;
    const u32x4 nan = {0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu};
    *reinterpret_cast<u32x4*>(out + j * (a.head_dim * 2)) = ok ? w[j] : nan;
  }
}

int row_lanes(int head_dim) {
  return head_dim <= 32 ? 4 : head_dim <= 64 ? 8 : head_dim <= 128 ? 16 : 32;
}

// Groups of a token's heads of one kind.
int64_t parts_of(int64_t heads) { return (heads + kRowsPer - 1) / kRowsPer; }

template <template <int, bool, int> class Kernel, typename Args>
hipError_t launch_rows(const Args& a, int64_t tokens, int64_t parts, int head_dim, bool bf16,
                       int kind, hipStream_t stream) {
  const int lanes = row_lanes(head_dim);
  const int64_t groups = (tokens * parts * lanes + kRowThreads - 1) / kRowThreads;
  void (*kernel)(Args) = nullptr;
  auto pick = [&](auto lanes_t) {
    constexpr int kLanes = decltype(lanes_t)::value;
    switch (kind) {
      case 0: kernel = Kernel<kLanes, false, 0>::get(); break;
      case 1: kernel = Kernel<kLanes, true, 1>::get(); break;
      case 2: kernel = bf16 ? Kernel<kLanes, true, 2>::get() : Kernel<kLanes, false, 2>::get(); break;
      case 3: kernel = Kernel<kLanes, true, 3>::get(); break;
      default: break;
    }
  };
  switch (lanes) {
    case 4: pick(std::integral_constant<int, 4>{}); break;
    case 8: pick(std::integral_constant<int, 8>{}); break;
    case 16: pick(std::integral_constant<int, 16>{}); break;
    default: pick(std::integral_constant<int, 32>{}); break;
  }
  if (kernel == nullptr) return hipErrorInvalidValue;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(groups)), dim3(kRowThreads), 0, stream, a);
  return hipGetLastError();
}

template <int kLanes, bool kBf16, int kKind>
struct Write {
  static auto get() { return write_kernel<kLanes, kBf16, kKind>; }
};
template <int kLanes, bool kBf16, int kKind>
struct Read {
  static auto get() { return read_kernel<kLanes, kBf16, kKind>; }
};

}  // namespace

hipError_t launch_write_kv(const WriteArgs& a, bool bf16, int kind, hipStream_t stream) {
  return launch_rows<Write>(a, a.num_tokens, parts_of(a.num_q_heads) + 2 * parts_of(a.num_kv_heads),
                            a.head_dim, bf16, kind, stream);
}

hipError_t launch_read_kv(const ReadArgs& a, bool bf16, int kind, hipStream_t stream) {
  return launch_rows<Read>(a, a.num_tokens, 2 * parts_of(a.num_kv_heads), a.head_dim, bf16, kind,
                           stream);
}

}  // namespace vtoken
