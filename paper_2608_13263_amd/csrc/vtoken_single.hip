// Attention of one query per request over the paged cache (vtoken_paged_attention with
// max_queries 1): the decode step's call, with a sliding window and first tokens that stay visible.
//
//   single_kernel    one workgroup per (request, KV head, split): scores and the weighted sum of V
//                    of the query heads that share the KV head, on the matrix cores
//   shared_kernel    the same for up to four KV heads side by side, where a head's row is less than
//                    a line
//   codes_kernel     the same for 4-bit rows
//   single_combine   merges the splits (no launch where one covers every request)
//
// The keys that a query sees are its first min(sinks, ..) ones and its last `window`: a list whose
// entry t is slot t, or t + skip past the sinks, so that nothing hidden is read.
#include <math.h>

#include "vtoken_elements.h"

namespace vtoken {
namespace {

using namespace elements;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

// Bytes of a head's values in a row.
constexpr int head_bytes(int kind, int head_dim) {
  return kind <= 1 ? 2 * head_dim : kind == 2 ? head_dim : head_dim / 2;
}
// Tokens of a wave in a round: 4 KiB of K, and of V, but 16 to 64 (fp8: 128).
constexpr int wave_tokens(int kind, int head_dim) {
  const int t = 4096 / head_bytes(kind, head_dim);
  const int most = kind == 2 ? 128 : 64;
  return t < 16 ? 16 : t > most ? most : t;
}

// What a request's one query sees.
struct View {
  int64_t row;   // of q and out
  int ql;        // queries the request has (0: none; more than 1: outputs are NaN)
  int s0, n;
  int sk, skip, count;
  bool fixed;    // no slot is read: the outputs are zeros (no slots) or NaN
};
__device__ __forceinline__ View view_of(const PromptArgs& a, int r) {
  View v;
  v.s0 = a.slot_indptr[r];
  v.n = a.slot_count != nullptr ? a.slot_count[r] : a.slot_indptr[r + 1] - v.s0;
  v.row = r;
  v.ql = 1;
  if (a.q_indptr != nullptr) {
    const int q0 = a.q_indptr[r], q1 = a.q_indptr[r + 1];
    v.row = q0;
    v.ql = q0 < 0 || q1 > a.num_queries || q1 < q0 ? 0 : q1 - q0;
  }
  v.fixed = v.s0 < 0 || v.n <= 0 || v.n > a.max_tokens || v.ql > 1;
  const int low = a.window > 0 ? max(v.n - a.window, 0) : 0;
  v.sk = min(a.sinks, low);
  v.skip = low - v.sk;
  v.count = v.n - v.skip;
  return v;
}

template <bool kBf16>
__device__ __forceinline__ f32x4 mfma16(u32x4 x, u32x4 y, f32x4 acc) {
  if constexpr (kBf16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x),
                                                   __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x),
                                                  __builtin_bit_cast(f16x8, y), acc, 0, 0, 0);
  }
}

// Two weights as 16-bit operands. bf16 takes them in two parts each, off by 2^-15 of a weight (one part
// by 2^-8, which showed in the output as much as its own rounding): the upper bits, cut off, so that no
// part is negative, and the rest; where V may hold infinities (kInfinities), the rest is 2^-20 of the
// weight at least, so that none of them is multiplied by zero. 16- and 8-bit rows pay 0 to 2% for the
// second part, 4-bit rows 1 to 4%. fp16 takes a weight once rounded, half a step of 2^-11.
struct Weights {
  uint32_t hi, lo;
};
template <bool kBf16, bool kInfinities>
__device__ __forceinline__ Weights weights_of(float x, float y) {
  Weights w{0, 0};
  if constexpr (kBf16) {
    const uint32_t u = __float_as_uint(x), v = __float_as_uint(y);
    w.hi = __builtin_amdgcn_perm(v, u, 0x07060302);
    float p = x - __uint_as_float(u & 0xffff0000u), q = y - __uint_as_float(v & 0xffff0000u);
    if (kInfinities) {
      p = fmaxf(p, x * 0x1p-20f);
      q = fmaxf(q, y * 0x1p-20f);
    }
    w.lo = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(p), static_cast<__bf16>(q)});
  } else {
    w.hi = __builtin_bit_cast(uint32_t, f16x2{static_cast<_Float16>(x), static_cast<_Float16>(y)});
  }
  return w;
}

// Combined with the values of lanes i ^ 16, i ^ 32 and i ^ 48.
template <bool kMax>
__device__ __forceinline__ float groups_reduce(float x) {
  const auto op = [](float p, float q) { return kMax ? fmaxf(p, q) : p + q; };
  uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(op(__uint_as_float(r[0]), __uint_as_float(r[1])));
  const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// The waves' sums of each of a workgroup's kHeads heads (wave w: head w % kHeads) into the outputs at
// `to`, or the split's records. mrg: LDS, [wave][query head][head_dim + 4] floats.
template <bool kBf16, int kD, int kHeads>
__device__ __forceinline__ void merge_waves(const PromptArgs& a, float* mrg, float m, float l,
                                            const f32x4 (&o)[kD / 16], int r, int h0, int split,
                                            int splits, int64_t to) {
  using Elem = typename Act<kBf16>::elem;
  typedef Elem Elem4 __attribute__((ext_vector_type(4)));
  constexpr int kRec = kD + 4;
  const int lane = threadIdx.x & 63, grp = lane >> 4, row = lane & 15;
  const int G = a.group;
  if (row < G) {
    float* rec = mrg + ((threadIdx.x >> 6) * 16 + row) * kRec;
    if (grp == 0) {
      rec[0] = m;
      rec[1] = l;
    }
#pragma unroll
    for (int dc = 0; dc < kD / 16; ++dc) {
      *reinterpret_cast<f32x4*>(rec + 4 + dc * 16 + 4 * grp) = o[dc];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kHeads * G * (kD / 4); i += kThreads) {
    const int g = i / (kD / 4), d = i % (kD / 4) * 4;   // query head of the workgroup's
    const float* first = mrg + (g / G * 16 + g % G) * kRec;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; w += kHeads) top = fmaxf(top, first[w * 16 * kRec]);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; w += kHeads) {
      const float* wr = first + w * 16 * kRec;
      // (no wave is left out: a NaN or an infinity in the sums of one far below the others has to
      // reach the row, also times zero; one without a maximum holds zeros, or NaN)
      const float f = wr[0] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(wr[0] - top);
      x += *reinterpret_cast<const f32x4*>(wr + 4 + d) * f;
      total += wr[1] * f;
    }
    if (splits == 1) {
      const f32x4 y = x * (total == 0.f ? 0.f : 1.f / total);
      *reinterpret_cast<Elem4*>(reinterpret_cast<Elem*>(a.out) + to + g * kD + d) =
          Elem4{static_cast<Elem>(y.x), static_cast<Elem>(y.y), static_cast<Elem>(y.z),
                static_cast<Elem>(y.w)};
      continue;
    }
    float* rec = a.workspace +
                 (((int64_t)r * a.num_kv_heads * G + h0 * G + g) * splits + split) * (kD + 2);
    *reinterpret_cast<f32x4_in*>(rec + 2 + d) = x;
    if (d == 0) *reinterpret_cast<f32x2_in*>(rec) = f32x2{top, total};
  }
}

// Wave w takes a round's tokens w kIT .. on; the waves share nothing until the end, so that no barrier
// stands between a load and its use, and each has a round of K and of V (4 KiB each) in flight. The query
// heads of the KV head are the 16 columns of the products: K and V are read once for all of them.
// The sum of the weights is that before they become operands (weights_of).
//
// Bound: HBM. 64 requests, a window of 2,048 and 4 sinks, 8 KV heads of 128, 16 bits, 539 MB: 95 us,
// 5.7 TB/s (with the merge 100.6, 5.4), where reads alone reach 7.2. Loads that
// leave the caches alone (nontemporal) are for rows that no other workgroup reads.
template <bool kBf16, int kKind, int kD>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(kD > 128 ? 2 : 3)))
void single_kernel(PromptArgs a, int split_tokens, int splits) {
  using Elem = typename Act<kBf16>::elem;
  constexpr int kRow = head_bytes(kKind, kD);
  static_assert(kRow >= 128 && kKind <= 2, "whole lines");
  constexpr int kIT = wave_tokens(kKind, kD);
  constexpr int kStep = kWaves * kIT;                // tokens of a round
  constexpr int kTiles = kIT / 16;                   // 16-token score tiles
  constexpr int kChunks = kD / 32;                   // score k-steps
  constexpr int kKC = (kTiles + 1) / 2;              // 32-token value k-steps
  constexpr int kDC = kD / 16;                       // 16-element value chunks
  constexpr int kLanes = kRow / 16;                  // loads: lanes per token row
  constexpr int kTok = 64 / kLanes;                  // loads: tokens per instruction
  constexpr int kLd = kIT / kTok;                    // loads per operand and round
  constexpr int kSR = (kIT + 63) / 64;               // slot registers
  constexpr int kWin = kIT < 32 ? kIT : 32;          // V rows staged per k-step
  constexpr int kPerWin = kWin / kTok;               // V loads per k-step
  constexpr int kRowK = kRow + 16;                   // LDS bytes per K row
  constexpr int kRowV = kD * 2;                      // and per V row (16-bit, swizzled)
  constexpr int kWinB = kIT * kRowK > kWin * kRowV ? kIT * kRowK : kWin * kRowV;
  constexpr int kRec = kD + 4;                       // merge: m, l, padding, kD values
  constexpr int kMergeB = kWaves * 16 * kRec * 4;
  constexpr int kLdsB = kWaves * kWinB > kMergeB ? kWaves * kWinB : kMergeB;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kLdsB];
  __shared__ u32x4 q_s[kChunks][64];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.group;
  const int H = a.num_kv_heads;
  const int gs = decode_grid_splits(splits);
  const int rs = blockIdx.x % gs + blockIdx.x / (gs * H) * gs;
  const int h = blockIdx.x / gs % H;
  const int r = rs / gs;
  const int split = rs - r * gs;
  if (r >= a.num_reqs || split >= splits) return;
  const View v = view_of(a, r);
  const int t0 = split * split_tokens;
  if (v.ql == 0) return;
  const int64_t to = v.row * a.out_stride + (int64_t)h * G * kD;
  if (v.fixed) {
    if (split != 0) return;
    const Elem fill = static_cast<Elem>(v.n == 0 && v.s0 >= 0 && v.ql == 1 ? 0.f
                                                                            : __builtin_nanf(""));
    for (int i = 0; i < v.ql; ++i) {
      for (int d = tid; d < G * kD; d += kThreads) {
        reinterpret_cast<Elem*>(a.out)[to + i * a.out_stride + d] = fill;
      }
    }
    return;
  }
  if (t0 >= v.count) return;
  const int nt = min(split_tokens, v.count - t0);
  const uint8_t* kplane = a.kv + (int64_t)(2 * a.layer) * a.plane_bytes;
  const uint8_t* vplane = kplane + a.plane_bytes;
  const int grp = lane >> 4;    // operand k-group / result row group
  const int row = lane & 15;    // token of a tile (K operand) / column (Q, P, results)
  const int wt0 = wave * kIT;   // this wave's first token of round 0
  const int rounds = wt0 < nt ? (nt - wt0 + kStep - 1) / kStep : 0;

  // Slots of round i: lane l holds token l (and l + 64) of the wave's; tokens past the split's end
  // re-read its last one
  struct Slots {
    int s[kSR];
  };
  auto load_slots = [&](int i) {
    Slots x;
#pragma unroll
    for (int q = 0; q < kSR; ++q) {
      const int t = t0 + min(wt0 + i * kStep + q * 64 + lane, nt - 1);
      x.s[q] = a.slots[(int64_t)v.s0 + t + (t < v.sk ? 0 : v.skip)];
    }
    return x;
  };
  bool bad = false;   // a slot outside the pool: never dereferenced, poisons the request
  int ls[kLd];        // slots of this lane's rows
  auto spread_slots = [&](Slots x) {
#pragma unroll
    for (int q = 0; q < kSR; ++q) {
      const bool ok = static_cast<unsigned>(x.s[q]) < static_cast<unsigned>(a.num_slots);
      bad |= !ok;
      x.s[q] = ok ? x.s[q] : 0;
    }
#pragma unroll
    for (int k = 0; k < kLd; ++k) {
      ls[k] = __shfl(x.s[k * kTok / 64], (k * kTok + lane / kLanes) & 63, 64);
    }
  };
  const int64_t lane0 = (int64_t)h * kRow + (lane % kLanes) * 16;
  auto load_rows = [&](const uint8_t* plane, u32x4 (&x)[kLd]) {
#pragma unroll
    for (int k = 0; k < kLd; ++k) {
      const u32x4* src = reinterpret_cast<const u32x4*>(plane + ((int64_t)ls[k] * a.row_bytes + lane0));
      x[k] = __builtin_nontemporal_load(src);
    }
  };
  Slots cur = load_slots(0);
  Slots nxt = load_slots(1);
  // The head dims of a k-chunk's lane group: any assignment gives the same dot products as long as
  // q and K use the same one. A lane's two pieces of fp8 of a pair of chunks are contiguous.
  constexpr bool kPair = kKind == 2;
  auto head_dim_of = [&](int ch) {
    return kPair ? (ch >> 1) * 64 + grp * 16 + (ch & 1) * 8 : ch * 32 + grp * 8;
  };
  const Elem* qrow = reinterpret_cast<const Elem*>(a.q) + v.row * a.q_stride +
                     (int64_t)(h * G + (row < G ? row : 0)) * kD;
  u32x4 qraw[(kChunks + kWaves - 1) / kWaves];
#pragma unroll
  for (int x = 0; x < (kChunks + kWaves - 1) / kWaves; ++x) {
    const int ch = min(wave + x * kWaves, kChunks - 1);
    qraw[x] = *reinterpret_cast<const u32x4*>(qrow + head_dim_of(ch));
  }
  u32x4 kr[kLd], vr[kLd];
  spread_slots(cur);
  load_rows(kplane, kr);
  load_rows(vplane, vr);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int x = 0; x < (kChunks + kWaves - 1) / kWaves; ++x) {
    if (wave + x * kWaves < kChunks) {
      u32x4 w = qraw[x];
      if (a.scale < 0.f) w ^= 0x80008000u;
      if (row >= G || a.scale == 0.f) w = u32x4{0, 0, 0, 0};
      q_s[wave + x * kWaves][lane] = w;
    }
  }
  __syncthreads();   // query operands in LDS; the K and V loads stay in flight
  // weights are powers of two, with a positive factor
  const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.44269504088896340736f;
  // this wave's window; only this wave touches it, and a wave's LDS operations run in order, so
  // a compiler fence is all that its reads of other lanes' writes need
  lds_u8* const win = (lds_u8*)lds + wave * kWinB;
  auto order_lds = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); };

  float m = -INFINITY, l = 0.f;
  f32x4 o[kDC];
#pragma unroll
  for (int dc = 0; dc < kDC; ++dc) o[dc] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto round = [&](int i, auto more_t) {
    constexpr bool kMore = decltype(more_t)::value;
    // ---- K rows into the window; the next round's K loads
    order_lds();
    {
      lds_u8* dst = win + (lane / kLanes) * kRowK + (lane % kLanes) * 16;
#pragma unroll
      for (int k = 0; k < kLd; ++k) *(lds_u32x4*)(dst + k * kTok * kRowK) = kr[k];
    }
    order_lds();
    if constexpr (kMore) {
      spread_slots(nxt);
      load_rows(kplane, kr);
      nxt = load_slots(i + 2);
    }
    __builtin_amdgcn_sched_barrier(0);

    u32x4 qop[kChunks];
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) qop[ch] = q_s[ch][lane];
    // ---- scores: lane holds tokens 16 t + 4*grp + j of its column's head
    f32x4 sc[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const lds_u8* src = win + (t * 16 + row) * kRowK;
      f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};   // two chains of products
      if constexpr (kPair) {
#pragma unroll
        for (int ch = 0; ch < kChunks; ch += 2) {
          const u32x4 w = *(const lds_u32x4*)(src + ch * 32 + grp * 16);
          acc[0] = mfma16<kBf16>(widen_fp8<kBf16>(u32x2{w.x, w.y}), qop[ch], acc[0]);
          acc[1] = mfma16<kBf16>(widen_fp8<kBf16>(u32x2{w.z, w.w}), qop[ch + 1], acc[1]);
        }
      } else {
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
          acc[ch & 1] = mfma16<kBf16>(
              *(const lds_u32x4*)(src + ch * 64 + grp * 16), qop[ch], acc[ch & 1]);
        }
      }
      sc[t] = acc[0] + acc[1];
    }
    const int left = nt - (wt0 + i * kStep);   // tokens of this round that exist
    if (left < kIT) {   // (uniform) the last round; a weight of zero would make an infinity of V a NaN
#pragma unroll
      for (int k = 0; k < kLd; ++k) {
        if (k * kTok + lane / kLanes >= left) vr[k] = u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (16 * t + 4 * grp + j >= left) sc[t][j] = -INFINITY;
        }
    }

    // ---- softmax weights per head (the four lanes of a column share m), powers of two of what a
    // score is above m (see Act)
    float top = sc[0][0];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, sc[t][j]);
    top = groups_reduce<true>(top) * scale;
    if (__ballot(top > m + Act<kBf16>::kMost) != 0) {
      const float next = fmaxf(top - Act<kBf16>::kFirst, m);
      const float f = next == m ? 1.f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int dc = 0; dc < kDC; ++dc) o[dc] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sc[t][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][j], scale, -base));
        l += sc[t][j];
      }

    // ---- O += V^T . P^T, one 32-token step at a time through the window
#pragma unroll
    for (int kc = 0; kc < kKC; ++kc) {
      order_lds();
#pragma unroll
      for (int k = 0; k < kPerWin; ++k) {
        const u32x4 w = vr[kc * kPerWin + k];
        const int tk = lane / kLanes + k * kTok, ln = lane % kLanes;
        if constexpr (kKind <= 1) {
          *(lds_u32x4*)(win + piece_at<kD>(tk, ln)) = w;
        } else {
          const int turn = write_turn<kKind, kD>(tk, ln);
          const uint32_t at = piece_at<kD>(tk, ln * 2 + turn);
          u32x4 out[2];
          widen<kBf16, kKind>(w, 0.f, turn, out);
          *(lds_u32x4*)(win + at) = out[0];
          *(lds_u32x4*)(win + (at ^ 16)) = out[1];
        }
      }
      order_lds();
      if constexpr (kMore) {
        if (kc == kKC - 1) {   // V is in the window: the next round's loads
          load_rows(vplane, vr);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      // P operand: tokens 4*grp..+3 of tile 2kc, then of tile 2kc+1; where there is one tile, its
      // weights' lower parts, by the same V rows
      u32x4 w = {0, 0, 0, 0}, w_lo = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int tile = 2 * kc + j / 2;
        if (tile >= kTiles) continue;
        const f32x4 p = sc[tile < kTiles ? tile : 0];
        const Weights x = weights_of<kBf16, kKind == 1>(p[j % 2 * 2], p[j % 2 * 2 + 1]);
        w[j] = x.hi;
        if (kTiles > 1) {
          w_lo[j] = x.lo;
        } else {
          w[j + 2] = x.lo;
        }
      }
      // V operand rows: lane 16*grp + rho supplies the row of token 4*grp + rho/4 of the first
      // tile (then of the second), elements 4*(rho%4)..+3 of the 16-element chunk
      // (piece 2 dc + .. of the row at r1 ^ 32 dc; 16 rows on the swizzle is the same)
      const uint32_t r1 = piece_at<kD>(4 * grp + row / 4, row >> 1 & 1) + (row & 1) * 8;
#pragma unroll
      for (int dc = 0; dc < kDC; ++dc) {
        const i16x4 x1 = lds_read_tr16(win + (r1 ^ (dc << 5)));
        i16x4 x2 = kBf16 ? x1 : i16x4{0, 0, 0, 0};
        if constexpr (kTiles > 1) x2 = lds_read_tr16(win + (r1 ^ (dc << 5)) + 16 * kRowV);
        const i16x8 xv = {x1[0], x1[1], x1[2], x1[3], x2[0], x2[1], x2[2], x2[3]};
        o[dc] = mfma16<kBf16>(__builtin_bit_cast(u32x4, xv), w, o[dc]);
        if (kBf16 && kTiles > 1) o[dc] = mfma16<kBf16>(__builtin_bit_cast(u32x4, xv), w_lo, o[dc]);
      }
    }
  };
  for (int i = 0; i + 1 < rounds; ++i) round(i, std::true_type{});
  if (rounds > 0) round(rounds - 1, std::false_type{});

  // ---- merge the waves: [m, l] and O[head][d] per wave into LDS
  l = groups_reduce<false>(l);
  if (__ballot(bad) != 0 && rounds > 0) l = __builtin_nanf("");
  __syncthreads();  // the windows are reused for the merge
  merge_waves<kBf16, kD, 1>(a, reinterpret_cast<float*>(lds), m, l, o, r, h, split, splits, to);
}

// kBytes bytes of a cache row (a power of two; aligned to that, or to 16).
template <int kBytes>
struct Exponents {
  u32x4 w[(kBytes + 15) / 16];
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) w[i] = *reinterpret_cast<const u32x4*>(p + 16 * i);
    } else if constexpr (kBytes == 8) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(p);
      w[0].x = x.x;
      w[0].y = x.y;
    } else {
      w[0].x = kBytes == 4   ? *reinterpret_cast<const uint32_t*>(p)
               : kBytes == 2 ? *reinterpret_cast<const uint16_t*>(p)
                             : *p;
    }
  }
  __device__ __forceinline__ void fetch(const lds_u8* p) {
    static_assert(kBytes <= 8, "a head's");
    if constexpr (kBytes == 8) {
      const u32x2 x = *(const lds_u32x2*)p;
      w[0].x = x.x;
      w[0].y = x.y;
    } else {
      w[0].x = kBytes == 4 ? *(const lds_u32*)p : kBytes == 2 ? *(const lds_u16*)p : *p;
    }
  }
  __device__ __forceinline__ void store(lds_u8* p) const {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) *(lds_u32x4*)(p + 16 * i) = w[i];
    } else if constexpr (kBytes == 8) {
      *(lds_u32x2*)p = u32x2{w[0].x, w[0].y};
    } else if constexpr (kBytes == 4) {
      *(lds_u32*)p = w[0].x;
    } else if constexpr (kBytes == 2) {
      *(lds_u16*)p = static_cast<uint16_t>(w[0].x);
    } else {
      *p = static_cast<uint8_t>(w[0].x);
    }
  }
};

typedef int i32x8 __attribute__((ext_vector_type(8)));

// 16 tokens x 128 head dims x 16 columns of 4-bit K as it is stored, a lane's 32 codes (one exponent's)
// of token lane % 16, by 8-bit queries with an exponent of their own per lane.
__device__ __forceinline__ f32x4 mfma_codes(u32x4 k, uint32_t k_exp, i32x8 q, uint32_t q_exp,
                                            f32x4 acc) {
  const i32x8 x = {static_cast<int>(k.x), static_cast<int>(k.y), static_cast<int>(k.z),
                   static_cast<int>(k.w), 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, q, acc, 4, 0, 0,
                                                          static_cast<int>(k_exp), 0,
                                                          static_cast<int>(q_exp));
}

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// bf16 query values as two e4m3 parts each, x = (hi + lo) 2^(e - 127): the upper four and the lower four
// of a value's eight bits; exact for values down to 2^-9 of the largest, to 2^-17 of it below.
template <int kN>
__device__ __forceinline__ void query_parts(const u32x4 (&w)[kN][4], float most, i32x8 (&hi)[kN],
                                            i32x8 (&lo)[kN], uint32_t& e) {
  e = max((__float_as_int(most) >> 23) - 7, 1);   // the largest becomes 128 to 256
  const float inverse = __int_as_float((254 - e) << 23);
#pragma unroll
  for (int x = 0; x < kN; ++x)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float y[4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t u = w[x][i / 2][i % 2 * 2 + j];
        y[2 * j] = __uint_as_float(u << 16) * inverse;
        y[2 * j + 1] = __uint_as_float(u & 0xffff0000u) * inverse;
      }
      int h = 0, r = 0;
      h = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], h, false);
      h = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], h, true);
      const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(h, false);
      const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(h, true);
      r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] - a.x, y[1] - a.y, r, false);
      r = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] - b.x, y[3] - b.y, r, true);
      hi[x][i] = h;
      lo[x][i] = r;
    }
}

template <bool kBf16>
__device__ __forceinline__ f32x4 mfma16x16(i16x4 x, i16x4 y, f32x4 acc) {
  if constexpr (kBf16) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(x, y, acc, 0, 0, 0);
  } else {
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4, x),
                                                 __builtin_bit_cast(f16x4, y), acc, 0, 0, 0);
  }
}

// LDS of shared_kernel: the round's K and V rows as stored, a window of widened V rows per wave.
constexpr int shared_window(int kind, int head_dim) {   // rows
  const int pieces = head_bytes(kind, head_dim) / 16;
  return pieces < 4 ? 64 / pieces : 16;
}
constexpr int shared_lds_bytes(int kind, int head_dim, int heads) {
  const int step = wave_tokens(kind, head_dim) * kWaves / heads;
  return 2 * step * (head_bytes(kind, head_dim) * heads + 16) +
         kWaves * shared_window(kind, head_dim) * head_dim * 2;
}

// Head rows of less than a line (an 8-bit head of 64 dims, 8 KV heads, 32 requests of 4,096 tokens: 37 us,
// 3.7 TB/s, where single_kernel's pieces of half lines take 54; a 16-bit head of 32 dims 33 instead of 52;
// with one KV head, or few tokens, both take the same). Wave w takes head w % kHeads of the workgroup's kHeads, and of a
// round's tokens the (w / kHeads)-th kIT; the workgroup loads the round's rows together, whole lines
// of all its heads at a time, and passes them through LDS as they are stored.
template <bool kBf16, int kKind, int kD, int kHeads>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(
    kD > 128 || shared_lds_bytes(kKind, kD, kHeads) > 160 * 1024 / 3 ? 2 : 3)))
void shared_kernel(PromptArgs a, int split_tokens, int splits) {
  using Elem = typename Act<kBf16>::elem;
  constexpr int kRow = head_bytes(kKind, kD);        // bytes of a head's row
  constexpr int kIT = wave_tokens(kKind, kD);        // tokens of a wave in a round
  constexpr int kTG = kWaves / kHeads;               // waves of a head
  constexpr int kStep = kIT * kTG;                   // tokens of a round
  constexpr int kTW = kStep / kWaves;                // of which a wave loads
  constexpr int kLanes = kRow * kHeads / 16;         // loads: lanes per token
  constexpr int kTok = 64 / kLanes;                  // and tokens per instruction
  constexpr int kLd = kTW / kTok;
  constexpr int kSR = (kTW + 63) / 64;
  constexpr int kRaw = kRow * kHeads + 16;           // LDS bytes of a token as stored
  constexpr int kTiles = kIT / 16;
  constexpr int kChunks = kD / 32;                   // score k-steps (1 or 2; not of codes)
  constexpr int kDC = kD / 16;
  constexpr int kPieces = kRow / 16;                 // 16-byte pieces of a head's row
  constexpr int kWin = shared_window(kKind, kD);             // V rows widened at a time
  constexpr int kPer = kWin * kPieces / 64;          // pieces of a lane per window
  constexpr int kRec = kD + 4;
  constexpr int kRawB = kStep * kRaw;
  constexpr int kWinB = kWin * kD * 2;
  constexpr int kUse = shared_lds_bytes(kKind, kD, kHeads);
  static_assert(kUse == 2 * kRawB + kWaves * kWinB && kKind <= 2, "LDS");
  constexpr int kMergeB = kWaves * 16 * kRec * 4;
  static_assert(kLd * kTok == kTW && kPer * 64 == kWin * kPieces && kIT % kWin == 0, "geometry");
  __shared__ __attribute__((aligned(16))) uint8_t lds[kUse > kMergeB ? kUse : kMergeB];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hw = wave % kHeads, tg = wave / kHeads;
  const int G = a.group;
  const int H = a.num_kv_heads;
  const int HG = H / kHeads;
  const int gs = decode_grid_splits(splits);
  // head groups that share lines run on one XCD, eight workgroups apart
  const int oct = blockIdx.x / (8 * HG);
  const int in_oct = blockIdx.x - oct * 8 * HG;
  const int rs = oct * 8 + in_oct % 8;
  const int h0 = in_oct / 8 * kHeads;
  const int r = rs / gs;
  const int split = rs - r * gs;
  if (r >= a.num_reqs || split >= splits) return;
  const View v = view_of(a, r);
  const int t0 = split * split_tokens;
  if (v.ql == 0) return;
  const int64_t to = v.row * a.out_stride + (int64_t)h0 * G * kD;   // the workgroup's heads
  if (v.fixed) {
    if (split != 0) return;
    const Elem fill = static_cast<Elem>(v.n == 0 && v.s0 >= 0 && v.ql == 1 ? 0.f
                                                                            : __builtin_nanf(""));
    for (int i = 0; i < v.ql; ++i) {
      for (int d = tid; d < kHeads * G * kD; d += kThreads) {
        reinterpret_cast<Elem*>(a.out)[to + i * a.out_stride + d] = fill;
      }
    }
    return;
  }
  if (t0 >= v.count) return;
  const int nt = min(split_tokens, v.count - t0);
  const int rounds = (nt + kStep - 1) / kStep;
  const uint8_t* kplane = a.kv + (int64_t)(2 * a.layer) * a.plane_bytes;
  const uint8_t* vplane = kplane + a.plane_bytes;
  const int grp = lane >> 4;    // operand k-group / result row group
  const int row = lane & 15;    // token of a tile (K operand) / column (Q, P, results)

  // slots of the tokens that this wave loads; those past the split's end re-read its last one
  struct Slots {
    int s[kSR];
  };
  const int32_t* slots = a.slots + v.s0;
  auto load_slots = [&](int i) {
    Slots x;
#pragma unroll
    for (int q = 0; q < kSR; ++q) {
      const int in_wave = kTW < 64 ? lane % kTW : q * 64 + lane;
      const int t = t0 + min(i * kStep + wave * kTW + in_wave, nt - 1);
      x.s[q] = slots[t + (t < v.sk ? 0 : v.skip)];
    }
    return x;
  };
  bool bad = false;   // a slot outside the pool: never dereferenced, poisons the request
  u32x4 kr[kLd], vr[kLd];
  const uint32_t row_bytes = static_cast<uint32_t>(a.row_bytes);
  auto load_rows = [&](Slots x) {
#pragma unroll
    for (int q = 0; q < kSR; ++q) {
      const bool ok = static_cast<unsigned>(x.s[q]) < static_cast<unsigned>(a.num_slots);
      bad |= !ok;
      x.s[q] = ok ? x.s[q] : 0;
    }
#pragma unroll
    for (int k = 0; k < kLd; ++k) {
      const uint32_t slot = __shfl(x.s[k * kTok / 64], (k * kTok + lane / kLanes) & 63, 64);
      const uint64_t at = (uint64_t)slot * row_bytes + h0 * kRow + (lane % kLanes) * 16;
      kr[k] = *reinterpret_cast<const u32x4*>(kplane + at);
      vr[k] = *reinterpret_cast<const u32x4*>(vplane + at);
    }
  };

  Slots nxt = load_slots(0);
  // ---- the query operand of the wave's head (any assignment of head dims to chunks gives the same
  // products as long as K has it too: a lane's piece of K is contiguous in its row)
  u32x4 q[kChunks];
  {
    const Elem* src = reinterpret_cast<const Elem*>(a.q) + v.row * a.q_stride +
                      (int64_t)((h0 + hw) * G + (row < G ? row : 0)) * kD;
#pragma unroll
    for (int ch = 0; ch < kChunks; ++ch) {
      q[ch] = *reinterpret_cast<const u32x4*>(
          src + (kKind == 2 ? grp * (kChunks > 1 ? 16 : 8) + ch * 8 : grp * 8));
      if (a.scale < 0.f) q[ch] ^= 0x80008000u;
      if (row >= G || a.scale == 0.f) q[ch] = u32x4{0, 0, 0, 0};
    }
  }
  load_rows(nxt);
  nxt = load_slots(1);
  // weights are powers of two, with a positive factor
  const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.44269504088896340736f;
  lds_u8* const kraw = (lds_u8*)lds;
  lds_u8* const vraw = kraw + kRawB;
  lds_u8* const win = vraw + kRawB + wave * kWinB;
  auto order_lds = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); };

  float m = -INFINITY, l = 0.f;
  f32x4 o[kDC];
#pragma unroll
  for (int dc = 0; dc < kDC; ++dc) o[dc] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int i = 0; i < rounds; ++i) {
    // ---- the round's rows to LDS, where the last round's have been read (its second barrier)
    {
      const uint32_t at = (wave * kTW + lane / kLanes) * kRaw + lane % kLanes * 16;
      const int left = nt - i * kStep - wave * kTW;   // rows of this wave's that exist
      if (left < kTW) {   // (a weight of zero would make an infinity of V a NaN)
#pragma unroll
        for (int k = 0; k < kLd; ++k) {
          if (k * kTok + lane / kLanes >= left) vr[k] = u32x4{0, 0, 0, 0};
        }
      }
#pragma unroll
      for (int k = 0; k < kLd; ++k) {
        *(lds_u32x4*)(kraw + at + k * kTok * kRaw) = kr[k];
        *(lds_u32x4*)(vraw + at + k * kTok * kRaw) = vr[k];
      }
    }
    __syncthreads();
    if (i + 1 < rounds) {
      load_rows(nxt);
      nxt = load_slots(i + 2);
    }
    // ---- scores: lane holds tokens 16 t + 4*grp + j of its column's head
    const int base_tok = tg * kIT;
    f32x4 sc[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int tk = base_tok + t * 16 + row;
      const lds_u8* src = kraw + tk * kRaw + hw * kRow;
      f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};   // two chains of products
      if constexpr (kKind == 2) {
        if constexpr (kChunks > 1) {
          const u32x4 w = *(const lds_u32x4*)(src + grp * 16);
          acc[0] = mfma16<kBf16>(widen_fp8<kBf16>(u32x2{w.x, w.y}), q[0], acc[0]);
          acc[1] = mfma16<kBf16>(widen_fp8<kBf16>(u32x2{w.z, w.w}), q[kChunks - 1], acc[1]);
          sc[t] = acc[0] + acc[1];
        } else {
          sc[t] = mfma16<kBf16>(widen_fp8<kBf16>(*(const lds_u32x2*)(src + grp * 8)), q[0], acc[0]);
        }
      } else {
        sc[t] = mfma16<kBf16>(*(const lds_u32x4*)(src + grp * 16), q[0], acc[0]);
      }
    }
    const int left = nt - (i * kStep + base_tok);   // tokens of the wave's round that exist
    if (left < kIT) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (16 * t + 4 * grp + j >= left) sc[t][j] = -INFINITY;
        }
    }
    // ---- softmax weights, as in single_kernel
    float top = sc[0][0];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, sc[t][j]);
    top = groups_reduce<true>(top) * scale;
    if (__ballot(top > m + Act<kBf16>::kMost) != 0) {
      const float next = fmaxf(top - Act<kBf16>::kFirst, m);
      const float f = next == m ? 1.f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int dc = 0; dc < kDC; ++dc) o[dc] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m;
    i16x4 w[kTiles], w_lo[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sc[t][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][j], scale, -base));
        l += sc[t][j];
      }
      const Weights x = weights_of<kBf16, kKind == 1>(sc[t][0], sc[t][1]);
      const Weights y = weights_of<kBf16, kKind == 1>(sc[t][2], sc[t][3]);
      w[t] = __builtin_bit_cast(i16x4, u32x2{x.hi, y.hi});
      w_lo[t] = __builtin_bit_cast(i16x4, u32x2{x.lo, y.lo});
    }
    // ---- O += V^T . P^T, a window of V rows at a time
#pragma unroll
    for (int y = 0; y < kIT / kWin; ++y) {
      u32x4 vw[kPer];
#pragma unroll
      for (int x = 0; x < kPer; ++x) {
        const int tk = base_tok + y * kWin + (x * 64 + lane) / kPieces, ln = lane % kPieces;
        vw[x] = *(const lds_u32x4*)(vraw + tk * kRaw + hw * kRow + ln * 16);
      }
      if (y == kIT / kWin - 1) __syncthreads();   // the round's rows have been read
      order_lds();
#pragma unroll
      for (int x = 0; x < kPer; ++x) {
        const int tk = (x * 64 + lane) / kPieces, ln = lane % kPieces;
        if constexpr (kKind <= 1) {
          *(lds_u32x4*)(win + piece_at<kD>(tk, ln)) = vw[x];
        } else {
          const int turn = write_turn<kKind, kD>(tk, ln);
          const uint32_t at = piece_at<kD>(tk, ln * 2 + turn);
          u32x4 out[2];
          widen<kBf16, kKind>(vw[x], 0.f, turn, out);
          *(lds_u32x4*)(win + at) = out[0];
          *(lds_u32x4*)(win + (at ^ 16)) = out[1];
        }
      }
      order_lds();
      // V operand rows: lane 16*grp + rho supplies the row of token 4*grp + rho/4, elements
      // 4*(rho%4)..+3 of the 16-element chunk
      const uint32_t r1 = piece_at<kD>(4 * grp + row / 4, row >> 1 & 1) + (row & 1) * 8;
#pragma unroll
      for (int t = 0; t < kWin / 16; ++t)
#pragma unroll
        for (int dc = 0; dc < kDC; ++dc) {
          const i16x4 x = lds_read_tr16(win + (r1 ^ (dc << 5)) + t * 16 * kD * 2);
          o[dc] = mfma16x16<kBf16>(x, w[y * (kWin / 16) + t], o[dc]);
          if (kBf16) o[dc] = mfma16x16<kBf16>(x, w_lo[y * (kWin / 16) + t], o[dc]);
        }
    }
  }

  // ---- merge the waves of each head: [m, l] and O[query head][d] per wave into LDS
  l = groups_reduce<false>(l);
  if (__syncthreads_or(bad) != 0) l = __builtin_nanf("");   // (the buffers are reused for the merge)
  merge_waves<kBf16, kD, kHeads>(a, reinterpret_cast<float*>(lds), m, l, o, r, h0, split, splits, to);
}

// 4-bit rows. Wave w takes head w % kHeads of the workgroup's kHeads and, of a round's tokens, the
// (w / kHeads)-th kIT; the workgroup loads the round's rows together, the pieces of all its heads of a
// token side by side, and passes them through LDS as they are stored.
//
//   scores   K stays as it is stored: 16 bytes of codes, 32 head dims of one token with one
//            exponent, are a lane's operand of a 16 tokens x 128 dims product of 4-bit by 8-bit
//            numbers with exponents (MFMA 16x16x128). The query's bf16 values go in as two e4m3
//            parts (see query_parts). Heads of fewer dims leave blocks of the 128 over: a lane group
//            past the head's pieces holds those of the next tiles, and a query in the blocks of one
//            tile, zeros in the others, picks that tile.
//   values   come back from LDS transposed as codes (ds_read_b64_tr_b4: a lane gets one head dim of 16
//            tokens). They multiply as bf16 without their exponents, which differ from token to
//            token and so go to the weights: w 2^(e - 127), exact, one set of weights (two parts each)
//            per 32 dims, formed for 32 tokens at a time (for 64 at once the kernel took 12 to 22% more).
//
// Bound: HBM and latency. 29 requests of 5,043 to 19,788 tokens, 8 KV heads of 128 with 8 query heads
// each, 411 MB: 105 to 108 us, 3.9 TB/s (112 to 114 with the merge, 3.6; with weights of one part the loads
// alone took 88 and the arithmetic alone 46). Widened to bf16 on their way into LDS, V took 48 LDS
// instructions per 64 tokens of 128 dims instead of 24, and K 64 conversions instead of none; with each wave
// loading for itself, its 64-byte pieces and 4-byte exponents came in at 3.5 TB/s with nothing else to do.
template <int kD, int kHeads>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(kD > 128 ? 2 : 3)))
void codes_kernel(PromptArgs a, int split_tokens, int splits) {
  constexpr int kRow = kD / 2;                       // bytes of a head's codes
  constexpr int kPieces = kD / 32;                   // 16-byte pieces, an exponent each
  constexpr int kIT = wave_tokens(3, kD);            // tokens of a wave in a round: 64, or 32
  constexpr int kStep = kIT * kWaves / kHeads;       // tokens of a round
  constexpr int kTW = kStep / kWaves;                // of which a wave loads
  constexpr int kLanes = kRow * kHeads / 16;         // loads: lanes per token
  constexpr int kTok = 64 / kLanes;                  // and tokens per instruction
  constexpr int kLd = kTW / kTok;
  constexpr int kTiles = kIT / 16;
  constexpr int kVar = kPieces < 4 ? 4 / kPieces : 1;     // tiles of a K read: queries in as many places
  constexpr int kBlk = kPieces > 4 ? kPieces / 4 : 1;     // 128-dim products of a tile
  constexpr int kKC = kIT / 32;                      // 32-token value k-steps
  constexpr int kDC = kD / 16;
  constexpr int kRec = kD + 4;
  constexpr int kRawK = kRow * kHeads + 16;          // LDS bytes of a token's codes: 16-byte reads
  constexpr int kRawV = kRow * kHeads + 8;           // of 16 tokens; 8-byte ones of 64
  constexpr int kExp = kPieces * kHeads;             // exponents of a token
  constexpr int kVAt = kStep * kRawK, kEAt = kVAt + kStep * kRawV, kScAt = kEAt + 2 * kStep * kExp;
  constexpr int kScB = kPieces * kIT * 4;
  constexpr int kUse = kScAt + kWaves * kScB, kMergeB = kWaves * 16 * kRec * 4;
  static_assert(kLd * kTok == kTW && kScAt % 16 == 0, "geometry");
  __shared__ __attribute__((aligned(16))) uint8_t lds[kUse > kMergeB ? kUse : kMergeB];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hw = wave % kHeads, tg = wave / kHeads;
  const int G = a.group;
  const int H = a.num_kv_heads;
  const int HG = H / kHeads;
  const int gs = decode_grid_splits(splits);
  // workgroups whose heads share lines run on one XCD, eight apart
  const int oct = blockIdx.x / (8 * HG);
  const int in_oct = blockIdx.x - oct * 8 * HG;
  const int rs = oct * 8 + in_oct % 8;
  const int h0 = in_oct / 8 * kHeads;
  const int r = rs / gs;
  const int split = rs - r * gs;
  if (r >= a.num_reqs || split >= splits) return;
  const View v = view_of(a, r);
  const int t0 = split * split_tokens;
  if (v.ql == 0) return;
  const int64_t to = v.row * a.out_stride + (int64_t)h0 * G * kD;   // the workgroup's heads
  if (v.fixed) {
    if (split != 0) return;
    const __bf16 fill = static_cast<__bf16>(v.n == 0 && v.s0 >= 0 && v.ql == 1
                                                ? 0.f
                                                : __builtin_nanf(""));
    for (int i = 0; i < v.ql; ++i) {
      for (int d = tid; d < kHeads * G * kD; d += kThreads) {
        reinterpret_cast<__bf16*>(a.out)[to + i * a.out_stride + d] = fill;
      }
    }
    return;
  }
  if (t0 >= v.count) return;
  const int nt = min(split_tokens, v.count - t0);
  const int wt0 = tg * kIT;     // the first token of a round that this wave computes
  const int rounds = (nt + kStep - 1) / kStep;
  const uint8_t* kplane = a.kv + (int64_t)(2 * a.layer) * a.plane_bytes;
  const uint8_t* vplane = kplane + a.plane_bytes;
  const int grp = lane >> 4;    // operand k-group / result row group
  const int row = lane & 15;    // token of a tile (K operand) / column (Q, P, results)

  // slot of the lane's token of those that this wave loads (lanes past them repeat); tokens past the
  // split's end re-read its last one
  const int32_t* slots = a.slots + v.s0;
  auto load_slot = [&](int i) {
    const int t = t0 + min(i * kStep + wave * kTW + lane % kTW, nt - 1);
    return slots[t + (t < v.sk ? 0 : v.skip)];
  };
  bool bad = false;   // a slot outside the pool: never dereferenced, poisons the request
  const uint32_t row_bytes = static_cast<uint32_t>(a.row_bytes);
  u32x4 kr[kLd], vr[kLd];
  Exponents<kExp> ke, ve;
  auto load_rows = [&](int s) {
    const bool ok = static_cast<unsigned>(s) < static_cast<unsigned>(a.num_slots);
    bad |= !ok;
    s = ok ? s : 0;
#pragma unroll
    for (int k = 0; k < kLd; ++k) {
      const uint32_t slot = __shfl(s, k * kTok + lane / kLanes, 64);
      const uint64_t at = (uint64_t)slot * row_bytes + h0 * kRow + lane % kLanes * 16;
      kr[k] = *reinterpret_cast<const u32x4*>(kplane + at);
      vr[k] = *reinterpret_cast<const u32x4*>(vplane + at);
    }
    const uint64_t at = (uint64_t)static_cast<uint32_t>(s) * row_bytes + H * kRow + h0 * kPieces;
    ke.load(kplane + at);
    ve.load(vplane + at);
  };

  int nxt = load_slot(0);
  // ---- the query: 8-bit operand, dims 16 grp .. + 15 and 64 + 16 grp .. of a 128-dim product's
  i32x8 q_hi[kBlk * kVar], q_lo[kBlk * kVar];
  uint32_t q_exp;
  {
    const uint16_t* src = reinterpret_cast<const uint16_t*>(a.q) + v.row * a.q_stride +
                          (int64_t)((h0 + hw) * G + (row < G ? row : 0)) * kD;
    const bool zero = row >= G || a.scale == 0.f;
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
    u32x4 w[kBlk * kVar][4];
    int top = 0;
#pragma unroll
    for (int x = 0; x < kBlk * kVar; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        // block of 32 dims of the product; with variants, x places the head's blocks from x pieces on
        const int block = 2 * (y / 2) + (grp >> 1);
        const int mine = kVar > 1 ? block - x * kPieces : x * 4 + block;
        const bool none = zero || mine < 0 || mine >= kPieces;
        w[x][y] = *reinterpret_cast<const u32x4*>(src + (none ? 0 : mine * 32) + (grp & 1) * 16 +
                                                  (y & 1) * 8);
        w[x][y] ^= sign;
        if (none) w[x][y] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          top = max(top, static_cast<int>(w[x][y][z] & 0x7fff0000u));
          top = max(top, static_cast<int>(w[x][y][z] << 16 & 0x7fff0000u));
        }
      }
    const float most = groups_reduce<true>(__int_as_float(top));   // over the query's dims
    query_parts(w, most, q_hi, q_lo, q_exp);
  }
  load_rows(nxt);
  nxt = load_slot(1);
  // weights are powers of two, with a positive factor
  const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.44269504088896340736f;
  lds_u8* const kraw = (lds_u8*)lds;
  lds_u8* const vraw = kraw + kVAt;
  lds_u8* const exps = kraw + kEAt;                    // [K, V][token][head][piece]
  lds_u8* const scales = kraw + kScAt + wave * kScB;   // of the wave's head, [piece][token] floats
  // a wave's LDS operations run in order: a compiler fence is all that reads of its own writes need
  auto order_lds = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); };

  float m = -INFINITY, l = 0.f;
  f32x4 o[kDC];
#pragma unroll
  for (int dc = 0; dc < kDC; ++dc) o[dc] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int i = 0; i < rounds; ++i) {
    // ---- the round's rows to LDS, where the last round's have been read (its second barrier)
#pragma unroll
    for (int k = 0; k < kLd; ++k) {
      const int tk = wave * kTW + k * kTok + lane / kLanes;
      *(lds_u32x4*)(kraw + tk * kRawK + lane % kLanes * 16) = kr[k];
      lds_u8* dst = vraw + tk * kRawV + lane % kLanes * 16;
      *(lds_u32x2*)dst = u32x2{vr[k].x, vr[k].y};
      *(lds_u32x2*)(dst + 8) = u32x2{vr[k].z, vr[k].w};
    }
    if (lane < kTW) {
      ke.store(exps + (wave * kTW + lane) * kExp);
      ve.store(exps + (kStep + wave * kTW + lane) * kExp);
    }
    __syncthreads();
    if (i + 1 < rounds) {
      load_rows(nxt);
      nxt = load_slot(i + 2);
    }
    // the exponents of V of the wave's tokens as powers of two
    if (lane < kIT) {
      typedef __attribute__((address_space(3))) float lds_float;
      Exponents<kPieces> e;
      e.fetch(exps + (kStep + wt0 + lane) * kExp + hw * kPieces);
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        *(lds_float*)(scales + (p * kIT + lane) * 4) = e8m0_scale(e.w[0][p / 4] >> (8 * (p % 4)) & 255);
      }
    }
    order_lds();
    // ---- scores: lane holds tokens 16 t + 4*grp + j of its column's head. Read x holds piece `grp`
    // (modulo the head's) of tile x kVar + grp / pieces, or, with more than four pieces, piece
    // grp + 4 (x % kBlk) of tile x / kBlk
    f32x4 sc[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < kTiles / kVar * kBlk; ++x) {
      const int tile = kPieces < 4 ? x * kVar + grp / kPieces : x / kBlk;
      const int pc = kPieces < 4 ? grp % kPieces : grp + x % kBlk * 4;
      const int tk = wt0 + 16 * tile + row;
      const u32x4 k = *(const lds_u32x4*)(kraw + tk * kRawK + hw * kRow + pc * 16);
      const uint32_t e = exps[tk * kExp + hw * kPieces + pc];
#pragma unroll
      for (int y = 0; y < kVar; ++y) {
        const int t = kVar > 1 ? x * kVar + y : x / kBlk;
        const int at_q = kVar > 1 ? y : x % kBlk;
        sc[t] = mfma_codes(k, e, q_hi[at_q], q_exp, sc[t]);
        sc[t] = mfma_codes(k, e, q_lo[at_q], q_exp, sc[t]);
      }
    }
    const int left = nt - (wt0 + i * kStep);   // tokens of the wave's round that exist
    if (left < kIT) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (16 * t + 4 * grp + j >= left) sc[t][j] = -INFINITY;
        }
    }
    // ---- softmax weights, as in single_kernel
    float top = sc[0][0];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, sc[t][j]);
    top = groups_reduce<true>(top) * scale;
    if (__ballot(top > m + Act<true>::kMost) != 0) {
      const float next = fmaxf(top - Act<true>::kFirst, m);
      const float f = next == m ? 1.f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int dc = 0; dc < kDC; ++dc) o[dc] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sc[t][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][j], scale, -base));
        l += sc[t][j];
      }
    // ---- O += V^T . P^T, 32 head dims at a time. Rows of a transpose read: the lane group's tokens
    // 16 t + 4 grp + j, t = 0 .. 3 of one 16-dim block, or t = 0, 1 of both blocks
    const int rho_tok = 16 * (row / 4 % kTiles) + 4 * grp + row % 4;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      auto codes = [&](int half) {   // of the piece
        return __builtin_amdgcn_ds_read_tr4_b64_v2i32(
            (lds_i32x2*)(vraw + (wt0 + rho_tok) * kRawV + hw * kRow + p * 16 + half * 8));
      };
      // codes of 8 tokens of head dim `row` of the piece's first 16 (x) and last (y), for each k-step
      const i32x2 x = codes(kKC == 2 ? 0 : row / 8);
      const i32x2 y = kKC == 2 ? codes(1) : x;
#pragma unroll
      for (int kc = 0; kc < kKC; ++kc) {
        u32x4 w, w_lo;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
          const f32x4 e =
              sc[2 * kc + z] * *(lds_f32x4*)(scales + (p * kIT + 16 * (2 * kc + z) + 4 * grp) * 4);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const Weights u = weights_of<true, false>(e[2 * j], e[2 * j + 1]);
            w[2 * z + j] = u.hi;
            w_lo[2 * z + j] = u.lo;
          }
        }
        const u32x4 v0 = widen_fp4(static_cast<uint32_t>(kKC == 2 ? x[kc] : x[0]), 1.f);
        const u32x4 v1 = widen_fp4(static_cast<uint32_t>(kKC == 2 ? y[kc] : x[1]), 1.f);
        o[2 * p] = mfma16<true>(v0, w, o[2 * p]);
        o[2 * p + 1] = mfma16<true>(v1, w, o[2 * p + 1]);
        o[2 * p] = mfma16<true>(v0, w_lo, o[2 * p]);
        o[2 * p + 1] = mfma16<true>(v1, w_lo, o[2 * p + 1]);
      }
    }
    __syncthreads();   // the round's rows have been read
  }

  // ---- merge the waves of each head: [m, l] and O[query head][d] per wave into LDS
  l = groups_reduce<false>(l);
  if (__syncthreads_or(bad) != 0) l = __builtin_nanf("");   // (the buffers are reused for the merge)
  merge_waves<true, kD, kHeads>(a, reinterpret_cast<float*>(lds), m, l, o, r, h0, split, splits, to);
}

// Merges the split records of one (request, query head). Bound: latency; the records are shared
// out over the waves, four in flight each.
template <bool kBf16, int kCW>
__global__ __launch_bounds__(64 * kCW) void single_combine(PromptArgs a, int split_tokens,
                                                           int splits) {
  using Elem = typename Act<kBf16>::elem;
  __shared__ float sum_s[kCW][256];
  const int heads = a.num_kv_heads * a.group;
  const int qh = blockIdx.x % heads;
  const int r = blockIdx.x / heads;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const View v = view_of(a, r);
  if (v.ql == 0 || v.fixed) return;   // (written by the first kernel)
  const int D = a.head_dim;
  const int64_t rs = D + 2;
  const int ns = min((v.count + split_tokens - 1) / split_tokens, splits);
  const float* rec0 = a.workspace + ((int64_t)r * heads + qh) * splits * rs;
  auto head_of = [&](int s) {
    return s < ns ? *reinterpret_cast<const f32x2_in*>(rec0 + s * rs) : f32x2{-INFINITY, 0.f};
  };
  const f32x2 first = head_of(lane);
  float top = first.x;
  for (int s = lane + 64; s < ns; s += 64) top = fmaxf(top, rec0[s * rs]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  float total = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
  for (int base = 0; base < ns; base += 64) {
    const f32x2 ml = base == 0 ? first : head_of(base + lane);
    // (as in merge_waves: every split counts, also one whose weight is zero)
    const float w = ml.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml.x - top);
    total += ml.y * w;
    for (int s = wave; s < 64 && base + s < ns; s += 4 * kCW) {
      float y[4][4], ws[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = s + j * kCW;
        const bool ok = t < 64 && base + t < ns;
        ws[j] = __shfl(w, t & 63, 64);
        const float* rec = rec0 + (ok ? base + t : base + s) * rs + 2;
#pragma unroll
        for (int c = 0; c < 4; ++c) y[j][c] = ok && c * 64 + lane < D ? rec[c * 64 + lane] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] += ws[j] * y[j][c];
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d, 64);
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if (c * 64 + lane < D) sum_s[wave][c * 64 + lane] = x[c];
  }
  __syncthreads();
  const float inv = total == 0.f ? 0.f : 1.f / total;
  Elem* dst = reinterpret_cast<Elem*>(a.out) + v.row * a.out_stride + (int64_t)qh * D;
  for (int d = tid; d < D; d += 64 * kCW) {
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < kCW; ++w) y += sum_s[w][d];
    dst[d] = static_cast<Elem>(y * inv);
  }
}

struct Splits {
  int tokens;   // of a split: a multiple of a round
  int count;    // of a request that sees as much as any may
};

// Whether a call takes shared_kernel, and for how many heads at a time.
bool takes_shared(int kind, int head_dim) { return kind == 3 || head_bytes(kind, head_dim) < 128; }
int shared_heads(int num_kv_heads) {
  return num_kv_heads % 4 == 0 ? 4 : num_kv_heads % 2 == 0 ? 2 : 1;
}

// Units of 32 KiB of K (at least a round) per split, by the estimate of decode_split_units(): the
// workgroups' rounds through the chip plus half a workgroup's time.
Splits single_splits(const PromptArgs& a, int kind) {
  const int heads = takes_shared(kind, a.head_dim) ? shared_heads(a.num_kv_heads) : 1;
  const int head = head_bytes(kind, a.head_dim);
  const int round = kWaves * wave_tokens(kind, a.head_dim) / heads;
  const int64_t unit_tokens = (32768 / (head * heads) + round - 1) / round * round;
  int64_t most = a.max_tokens;
  if (a.window > 0 && (int64_t)a.window + a.sinks < most) most = (int64_t)a.window + a.sinks;
  const int64_t pairs = (int64_t)a.num_reqs * (a.num_kv_heads / heads);
  const int resident = 256 * (a.head_dim > 128 ? 2 : 3);
  const double start = 3.0;
  const double unit = 2.0 * unit_tokens * head * heads * resident / 7e6;   // us
  Splits best{static_cast<int>(unit_tokens), 1};
  double best_time = 0;
  for (int u = 1; u <= 8; u *= 2) {
    const int64_t count = most > 0 ? (most + u * unit_tokens - 1) / (u * unit_tokens) : 1;
    const double one = start + u * unit;
    const double time = static_cast<double>(pairs * count) * one / resident + one / 2;
    if (u == 1 || time < best_time) {
      best = {static_cast<int>(u * unit_tokens), static_cast<int>(count)};
      best_time = time;
    }
  }
  return best;
}

using Kernel = void (*)(PromptArgs, int, int);

template <bool kBf16, int kKind, int kD>
Kernel pick(int num_kv_heads) {
  if constexpr (kKind == 3) {
    switch (shared_heads(num_kv_heads)) {
      case 4: return codes_kernel<kD, 4>;
      case 2: return codes_kernel<kD, 2>;
      default: return codes_kernel<kD, 1>;
    }
  } else if constexpr (head_bytes(kKind, kD) < 128) {
    switch (shared_heads(num_kv_heads)) {
      case 4: return shared_kernel<kBf16, kKind, kD, 4>;
      case 2: return shared_kernel<kBf16, kKind, kD, 2>;
      default: return shared_kernel<kBf16, kKind, kD, 1>;
    }
  } else {
    return single_kernel<kBf16, kKind, kD>;
  }
}

template <bool kBf16, int kKind>
Kernel pick_single(int head_dim, int num_kv_heads) {
  switch (head_dim) {
    case 32: return pick<kBf16, kKind, 32>(num_kv_heads);
    case 64: return pick<kBf16, kKind, 64>(num_kv_heads);
    case 128: return pick<kBf16, kKind, 128>(num_kv_heads);
    case 256: return pick<kBf16, kKind, 256>(num_kv_heads);
    default: return nullptr;
  }
}

// More splits, and rows that leave the chip room: 16 waves merge a row's records, else 4 (1,856 rows of
// 39: 16.7 us with 16, 8.7 with 4).
constexpr int kManySplits = 32, kManyRows = 1024;

}  // namespace

int64_t single_workspace_bytes(const PromptArgs& a, int kind) {
  const Splits s = single_splits(a, kind);
  if (s.count == 1) return 0;
  return (int64_t)a.num_reqs * a.num_kv_heads * a.group * s.count * (a.head_dim + 2) * 4;
}

hipError_t launch_single(const PromptArgs& a, bool bf16, int kind, hipStream_t stream) {
  const Splits s = single_splits(a, kind);
  const int heads = takes_shared(kind, a.head_dim) ? shared_heads(a.num_kv_heads) : 1;
  const int64_t groups = decode_grid_groups((int64_t)a.num_reqs * decode_grid_splits(s.count)) *
                         (a.num_kv_heads / heads);
  const int64_t rows = (int64_t)a.num_reqs * a.num_kv_heads * a.group;
  if (groups > UINT32_MAX / kThreads || rows > UINT32_MAX / 256) {   // (a grid's threads)
    return hipErrorInvalidValue;
  }
  Kernel kernel = nullptr;
  const int D = a.head_dim, H = a.num_kv_heads;
  switch (kind) {
    case 0: kernel = pick_single<false, 0>(D, H); break;
    case 1: kernel = pick_single<true, 1>(D, H); break;
    case 2: kernel = bf16 ? pick_single<true, 2>(D, H) : pick_single<false, 2>(D, H); break;
    case 3: kernel = pick_single<true, 3>(D, H); break;
    default: break;
  }
  if (kernel == nullptr) return hipErrorInvalidValue;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(groups)), dim3(kThreads), 0, stream, a,
                     s.tokens, s.count);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || s.count == 1) return e;
  const bool many = s.count > kManySplits && rows < kManyRows;
  const auto combine = bf16 ? (many ? single_combine<true, 16> : single_combine<true, 4>)
                            : (many ? single_combine<false, 16> : single_combine<false, 4>);
  hipLaunchKernelGGL(combine, dim3(static_cast<unsigned>(rows)), dim3(64 * (many ? 16 : 4)), 0,
                     stream, a, s.tokens, s.count);
  return hipGetLastError();
}

}  // namespace vtoken
