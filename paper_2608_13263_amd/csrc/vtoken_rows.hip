// Rows of the cache as values (vtoken_write_kv, vtoken_read_kv).
//
//   write_kernel   per-head RMS norm and rotation of q and k, k and v stored at their slots in the
//                  cache's type, q to its output
//   read_kernel    rows of listed slots widened to dense 16-bit tensors
//
// A head row is taken by a group of lanes, eight elements (16 bytes) each, so that a group reads
// its row with one load per lane, reduces and turns it in registers and stores it: every byte is
// moved once. Both are bound by HBM where the calls are large and by latency where they are small.
#include "vtoken_elements.h"

namespace vtoken {
namespace {

using namespace elements;

constexpr int kRowThreads = 256;

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
    top = max(top, __shfl_xor(top, 1, 64));
    top = max(top, __shfl_xor(top, 2, 64));
    const int field = top >> 23;
    const int e = field == 255 ? 255 : max(field - 2, 1);
    const float inverse = e == 255 ? 0.f : __int_as_float((254 - e) << 23);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = fabsf(x[i]) * inverse;   // exact but for what rounds to zero anyway
      const uint32_t code = (t > 0.25f) + (t >= 0.75f) + (t > 1.25f) + (t >= 1.75f) +
                            (t > 2.5f) + (t >= 3.5f) + (t > 5.f);
      const uint32_t sign = e != 255 && __float_as_int(x[i]) < 0 ? 8u : 0u;
      w |= (code | sign) << (4 * i);
    }
    *reinterpret_cast<uint32_t*>(row + h * (head_dim / 2) + sub * 4) = w;
    if ((sub & 3) == 0) {
      row[heads * (head_dim / 2) + h * (head_dim / 32) + sub / 4] = static_cast<uint8_t>(e);
    }
  }
}

// kLanes: lanes per head row (the power of two from head_dim / 8 on, at least 4).
template <int kLanes, bool kBf16, int kKind>
__global__ __launch_bounds__(kRowThreads) void write_kernel(WriteArgs a) {
  // the results decide roundings to 8 and 4 bits: no contraction, the formula's own roundings
#pragma clang fp contract(off)
  const int items = a.num_q_heads + 2 * a.num_kv_heads;   // head rows of a token: q, k, v
  const int64_t item = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) / kLanes;
  const int sub = threadIdx.x % kLanes;
  if (item >= (int64_t)a.num_tokens * items) return;
  const int t = static_cast<int>(item / items);
  const int i = static_cast<int>(item) - t * items;
  const int slot = a.slots[t];
  if (slot < 0) return;
  const bool is_q = i < a.num_q_heads;
  const bool is_v = i >= a.num_q_heads + a.num_kv_heads;
  const int h = is_q ? i : is_v ? i - a.num_q_heads - a.num_kv_heads : i - a.num_q_heads;
  const int D = a.head_dim;
  const int half = a.rotary_dim / 2;
  const bool mine = sub * 8 < D;
  const int pos = half > 0 ? a.positions[t] : 0;
  const bool bad = slot >= a.num_slots ||
                   (half > 0 && static_cast<unsigned>(pos) >= static_cast<unsigned>(a.num_positions));
  if (bad && !is_q) return;

  const uint8_t* src = is_q ? a.q : is_v ? a.v : a.k;
  const int64_t stride = is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride;
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (mine) {
    to_float<kBf16>(*reinterpret_cast<const u32x4*>(src + (t * stride + h * D + sub * 8) * 2), x);
  }
  if (!is_v) {
    const float* weight = is_q ? a.q_weight : a.k_weight;
    if (weight != nullptr) {
      double sum = 0.;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += static_cast<double>(x[j]) * x[j];
#pragma unroll
      for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor(sum, d, 64);
      const float r = static_cast<float>(1. / sqrt(sum / D + a.eps));
      if (mine) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] * r * weight[sub * 8 + j];
      }
    }
    if (half > 0) {
      const float* cs = a.cos_sin + (bad ? 0 : (int64_t)pos * a.rotary_dim);
      const int e = sub * 8;
      if (a.interleaved) {
        if (!bad && e < a.rotary_dim) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float c = cs[e / 2 + j], s = cs[half + e / 2 + j];
            const float p = x[2 * j], q = x[2 * j + 1];
            x[2 * j] = p * c - q * s;
            x[2 * j + 1] = q * c + p * s;
          }
        }
      } else {
        // the other half's values are half / 8 lanes on (or back)
        const int d = half / 8;
        const int from = (threadIdx.x & 63) + (e < half ? d : -d);
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = __shfl(x[j], from & 63, 64);
        if (!bad && e < a.rotary_dim) {
          const int at = e < half ? e : e - half;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float c = cs[at + j], s = cs[half + at + j];
            x[j] = e < half ? x[j] * c - y[j] * s : x[j] * c + y[j] * s;
          }
        }
      }
    }
  }
  if (!mine) return;
  if (is_q) {
    u32x4 w = to_act<kBf16>(x);
    if (bad) {
      float nan[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) nan[j] = __builtin_nanf("");
      w = to_act<kBf16>(nan);
    }
    *reinterpret_cast<u32x4*>(a.q_out + (t * a.q_out_stride + h * D + sub * 8) * 2) = w;
    return;
  }
  store_row<kBf16, kKind>((is_v ? a.vplane : a.kplane) + slot * a.row_bytes, a.num_kv_heads, D, h,
                          sub, x);
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
  const int items = 2 * a.num_kv_heads;
  const int64_t item = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) / kLanes;
  const int sub = threadIdx.x % kLanes;
  if (item >= (int64_t)a.num_tokens * items || sub * 8 >= a.head_dim) return;
  const int t = static_cast<int>(item / items);
  const int i = static_cast<int>(item) - t * items;
  const bool is_v = i >= a.num_kv_heads;
  const int h = is_v ? i - a.num_kv_heads : i;
  const int slot = a.slots[t];
  u32x4 w;
  if (static_cast<unsigned>(slot) < static_cast<unsigned>(a.num_slots)) {
    w = load_row<kBf16, kKind>((is_v ? a.vplane : a.kplane) + slot * a.row_bytes, a.num_kv_heads,
                               a.head_dim, h, sub);
  } else {
    float nan[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) nan[j] = __builtin_nanf("");
    w = to_act<kBf16>(nan);
  }
  *reinterpret_cast<u32x4*>((is_v ? a.v_out + t * a.v_stride * 2 : a.k_out + t * a.k_stride * 2) +
                            (h * a.head_dim + sub * 8) * 2) = w;
}

int row_lanes(int head_dim) {
  return head_dim <= 32 ? 4 : head_dim <= 64 ? 8 : head_dim <= 128 ? 16 : 32;
}

template <template <int, bool, int> class Kernel, typename Args>
hipError_t launch_rows(const Args& a, int64_t items, int head_dim, bool bf16, int kind,
                       hipStream_t stream) {
  const int lanes = row_lanes(head_dim);
  const int64_t groups = (items * lanes + kRowThreads - 1) / kRowThreads;
  if (groups > INT32_MAX) return hipErrorInvalidValue;
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
  return launch_rows<Write>(a, (int64_t)a.num_tokens * (a.num_q_heads + 2 * a.num_kv_heads),
                            a.head_dim, bf16, kind, stream);
}

hipError_t launch_read_kv(const ReadArgs& a, bool bf16, int kind, hipStream_t stream) {
  return launch_rows<Read>(a, (int64_t)a.num_tokens * 2 * a.num_kv_heads, a.head_dim, bf16, kind,
                           stream);
}

}  // namespace vtoken
