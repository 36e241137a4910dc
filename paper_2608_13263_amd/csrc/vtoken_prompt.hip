// Attention of a ragged batch of queries over the paged cache (vtoken_paged_attention): causal,
// with a sliding window and first tokens that stay visible, through a slot mapping.
//
//   simple_kernel   one wave per (query, query head): 64 keys at a time, running softmax
#include <math.h>

#include "vtoken_elements.h"

namespace vtoken {
namespace {

using namespace elements;

// One element of head h's row as a float.
template <int kKind>
__device__ __forceinline__ float element(const uint8_t* row, int heads, int head_dim, int h,
                                         int d) {
  if constexpr (kKind == 0) {
    return static_cast<float>(reinterpret_cast<const _Float16*>(row)[h * head_dim + d]);
  } else if constexpr (kKind == 1) {
    return static_cast<float>(reinterpret_cast<const __bf16*>(row)[h * head_dim + d]);
  } else if constexpr (kKind == 2) {
    return __builtin_amdgcn_cvt_f32_fp8(row[h * head_dim + d], 0);
  } else {
    const uint32_t code = row[(h * head_dim + d) / 2] >> (4 * (d & 1)) & 15;
    const float m = (code & 7) < 2 ? 0.5f * (code & 7)
                                   : __uint_as_float(((code & 7) / 2 + 126) << 23) *
                                         (code & 1 ? 1.5f : 1.f);
    return (code & 8 ? -m : m) *
           e8m0_scale(row[heads * (head_dim / 2) + (h * head_dim + d) / 32]);
  }
}

template <bool kBf16, int kKind>
__global__ __launch_bounds__(64) void simple_kernel(PromptArgs a) {
  using Elem = typename Act<kBf16>::elem;
  __shared__ float q_s[256];
  const int lane = threadIdx.x;
  const int heads = a.num_kv_heads * a.group;
  const int64_t id = blockIdx.x;
  const int qh = static_cast<int>(id % heads);
  const int i = static_cast<int>(id / heads % a.max_queries);
  const int r = static_cast<int>(id / heads / a.max_queries);
  const int q0 = a.q_indptr != nullptr ? a.q_indptr[r] : r;
  const int q1 = a.q_indptr != nullptr ? a.q_indptr[r + 1] : r + 1;
  if (q0 < 0 || q1 > a.num_queries || i >= q1 - q0) return;
  const int ql = q1 - q0;
  const int h = qh / a.group;
  const int D = a.head_dim;
  const int s0 = a.slot_indptr[r];
  const int n = a.slot_count != nullptr ? a.slot_count[r] : a.slot_indptr[r + 1] - s0;
  const bool fixed = s0 < 0 || n < 0 || n > a.max_tokens || ql > a.max_queries;
  const Elem* q = reinterpret_cast<const Elem*>(a.q);
  Elem* out = reinterpret_cast<Elem*>(a.out);
  for (int j = i; j < ql; j += a.max_queries) {   // more than one round only where ql is too large
    const int64_t at = (int64_t)(q0 + j) * a.q_stride + qh * D;
    const int64_t to = (int64_t)(q0 + j) * a.out_stride + qh * D;
    for (int d = lane; d < D; d += 64) q_s[d] = static_cast<float>(q[at + d]);
    __syncthreads();
    const uint8_t* kplane = a.kv + (int64_t)(2 * a.layer) * a.plane_bytes;
    const uint8_t* vplane = kplane + a.plane_bytes;
    const int64_t p = (int64_t)n - ql + j;
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t k0 = 0; !fixed && k0 <= p; k0 += 64) {
      const int64_t k = k0 + lane;
      const bool seen = k <= p && (a.window == 0 || k > p - a.window || k < a.sinks);
      if (__ballot(seen) == 0) continue;
      const int slot = seen ? a.slots[s0 + k] : 0;
      const bool bad = static_cast<unsigned>(slot) >= static_cast<unsigned>(a.num_slots);
      float x = -INFINITY;
      if (seen) {
        x = 0.f;
        const uint8_t* row = kplane + (bad ? 0 : slot) * a.row_bytes;
        for (int d = 0; d < D; ++d) x += q_s[d] * element<kKind>(row, a.num_kv_heads, D, h, d);
        x = bad ? __builtin_nanf("") : x * a.scale;
      }
      float mi = x;
      for (int d = 1; d < 64; d <<= 1) mi = fmaxf(mi, __shfl_xor(mi, d, 64));
      mi = fmaxf(mi, m);
      const float safe = mi == -INFINITY ? 0.f : mi;
      const float f = __expf(m - safe);
      m = mi;
      const float w = seen ? __expf(x - safe) : 0.f;
      l = l * f + w;
      for (int c = 0; c < 4; ++c) o[c] *= f;
      for (int t = 0; t < 64; ++t) {
        if (!__shfl(static_cast<int>(seen), t, 64)) continue;
        const float wt = __shfl(w, t, 64);
        const int st = __shfl(bad ? 0 : slot, t, 64);
        const uint8_t* row = vplane + st * a.row_bytes;
        for (int c = 0; c < 4; ++c) {
          if (c * 64 + lane < D) o[c] += wt * element<kKind>(row, a.num_kv_heads, D, h, c * 64 + lane);
        }
      }
    }
    for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d, 64);
    for (int c = 0; c < 4; ++c) {
      const int d = c * 64 + lane;
      if (d >= D) break;
      out[to + d] = static_cast<Elem>(fixed ? __builtin_nanf("") : l == 0.f ? 0.f : o[c] / l);
    }
    __syncthreads();
  }
}

}  // namespace

int64_t prompt_workspace_bytes(const PromptArgs& a, int kind) { return 0; }

hipError_t launch_prompt(const PromptArgs& a, bool bf16, int kind, hipStream_t stream) {
  const int64_t grid = (int64_t)a.num_reqs * a.max_queries * a.num_kv_heads * a.group;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  void (*kernel)(PromptArgs) = nullptr;
  switch (kind) {
    case 0: kernel = simple_kernel<false, 0>; break;
    case 1: kernel = simple_kernel<true, 1>; break;
    case 2: kernel = bf16 ? simple_kernel<true, 2> : simple_kernel<false, 2>; break;
    case 3: kernel = simple_kernel<true, 3>; break;
    default: return hipErrorInvalidValue;
  }
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(grid)), dim3(64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vtoken
