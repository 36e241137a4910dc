// Attention of one query per request over the paged cache (vtoken_paged_attention with
// max_queries 1): the decode step's call, with a sliding window and first tokens that stay visible.
//
//   single_kernel    one workgroup per (request, KV head, split): scores and the weighted sum of V
//                    of the query heads that share the KV head, on the matrix cores
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

template <bool kBf16, int kKind, int kD>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(kD > 128 ? 2 : 3)))
void single_kernel(PromptArgs a, int split_tokens, int splits) {
  using Elem = typename Act<kBf16>::elem;
  constexpr int kRow = head_bytes(kKind, kD);
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
  constexpr int kPerWin = kWin / kTok > 0 ? kWin / kTok : 1;   // V loads per k-step
  constexpr int kRowK = kRow + 16;                   // LDS bytes per K row
  constexpr int kRowV = kD * 2;                      // and per V row (16-bit, swizzled)
  constexpr int kWinB = kIT * kRowK > kWin * kRowV ? kIT * kRowK : kWin * kRowV;
  constexpr int kRec = kD + 4;                       // merge: m, l, padding, kD values
  constexpr int kMergeB = kWaves * 16 * kRec * 4;
  constexpr int kLdsB = kWaves * kWinB > kMergeB ? kWaves * kWinB : kMergeB;
  constexpr int kExp = kD / 32;                      // exponents of a head (4-bit rows)
  __shared__ __attribute__((aligned(16))) uint8_t lds[kLdsB];
  __shared__ u32x4 q_s[kChunks][64];
  __shared__ __attribute__((aligned(8))) uint8_t exp_s[kKind == 3 ? kWaves : 1][2][kIT][kExp];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.group;
  const int H = a.num_kv_heads;
  const int gs = decode_grid_splits(splits);
  int h, rs;
  if constexpr (kRow < 128) {
    // the heads of a split share the lines of their rows: they run on one XCD, eight workgroups
    // apart
    const int oct = blockIdx.x / (8 * H);
    const int x = blockIdx.x - oct * 8 * H;
    rs = oct * 8 + x % 8;
    h = x / 8;
  } else {
    rs = blockIdx.x % gs + blockIdx.x / (gs * H) * gs;
    h = blockIdx.x / gs % H;
  }
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
  int own = 0;        // slot of token `lane` (exponents)
  auto spread_slots = [&](Slots x) {
#pragma unroll
    for (int q = 0; q < kSR; ++q) {
      const bool ok = static_cast<unsigned>(x.s[q]) < static_cast<unsigned>(a.num_slots);
      bad |= !ok;
      x.s[q] = ok ? x.s[q] : 0;
    }
    own = x.s[0];
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
      if constexpr (kRow < 128) {
        x[k] = *src;   // its line is read by the other heads too
      } else {
        x[k] = __builtin_nontemporal_load(src);
      }
    }
  };
  // the head's exponents of token `lane`
  const int64_t exp0 = (int64_t)H * kRow + h * kExp;
  auto load_exp = [&](const uint8_t* plane) {
    const uint8_t* src = plane + ((int64_t)own * a.row_bytes + exp0);
    if constexpr (kExp == 8) {
      // two words: a head's eight exponents are aligned to eight bytes
      return *reinterpret_cast<const u32x2*>(src);
    } else if constexpr (kExp == 4) {
      return u32x2{*reinterpret_cast<const uint32_t*>(src), 0u};
    } else if constexpr (kExp == 2) {
      return u32x2{*reinterpret_cast<const uint16_t*>(src), 0u};
    } else {
      return u32x2{*src, 0u};
    }
  };
  auto put_exp = [&](uint8_t* dst, u32x2 x) {
    if constexpr (kExp == 8) {
      *reinterpret_cast<u32x2*>(dst) = x;
    } else if constexpr (kExp == 4) {
      *reinterpret_cast<uint32_t*>(dst) = x.x;
    } else if constexpr (kExp == 2) {
      *reinterpret_cast<uint16_t*>(dst) = static_cast<uint16_t>(x.x);
    } else {
      *dst = static_cast<uint8_t>(x.x);
    }
  };

  Slots cur = load_slots(0);
  Slots nxt = load_slots(1);
  // The head dims of a k-chunk's lane group: any assignment gives the same dot products as long as
  // q and K use the same one. A lane's pieces of fp8 (of a pair of chunks) and 4-bit rows (of all
  // of them) are contiguous.
  constexpr bool kPair = kKind == 2 && kChunks % 2 == 0;
  auto head_dim_of = [&](int ch) {
    return kKind == 3 ? grp * (kD / 4) + ch * 8
           : kPair    ? (ch >> 1) * 64 + grp * 16 + (ch & 1) * 8
                      : ch * 32 + grp * 8;
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
  u32x2 ke = {}, ve = {};
  spread_slots(cur);
  load_rows(kplane, kr);
  if constexpr (kKind == 3) ke = load_exp(kplane);
  load_rows(vplane, vr);
  if constexpr (kKind == 3) ve = load_exp(vplane);
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
      if constexpr (kKind == 3) {
        if (lane < kIT) {
          put_exp(exp_s[wave][0][lane], ke);
          put_exp(exp_s[wave][1][lane], ve);
        }
      }
    }
    order_lds();
    if constexpr (kMore) {
      spread_slots(nxt);
      load_rows(kplane, kr);
      if constexpr (kKind == 3) {
        ke = load_exp(kplane);
        ve = load_exp(vplane);
      }
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
      if constexpr (kKind == 3) {
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
          const uint32_t w = *(const lds_u32*)(src + grp * (kD / 8) + ch * 4);
          const float e = e8m0_scale(exp_s[wave][0][t * 16 + row][(grp * (kD / 4) + ch * 8) / 32]);
          acc[ch & 1] = mfma16<kBf16>(widen_fp4(w, e), qop[ch], acc[ch & 1]);
        }
      } else if constexpr (kPair) {
#pragma unroll
        for (int ch = 0; ch < kChunks; ch += 2) {
          const u32x4 w = *(const lds_u32x4*)(src + ch * 32 + grp * 16);
          acc[0] = mfma16<kBf16>(widen_fp8<kBf16>(u32x2{w.x, w.y}), qop[ch], acc[0]);
          acc[1] = mfma16<kBf16>(widen_fp8<kBf16>(u32x2{w.z, w.w}), qop[ch + 1], acc[1]);
        }
      } else if constexpr (kKind == 2) {
        acc[0] = mfma16<kBf16>(widen_fp8<kBf16>(*(const lds_u32x2*)(src + grp * 8)),
                               qop[0], acc[0]);
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
    if (left < kIT) {   // (uniform) the last round
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (16 * t + 4 * grp + j >= left) sc[t][j] = -INFINITY;
        }
    }

    // ---- softmax weights per head (the four lanes of a column share m), powers of two of what a
    // score is above m; m follows the maximum where that passes it by 2^8
    float top = sc[0][0];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, sc[t][j]);
    top = groups_reduce<true>(top) * scale;
    if (__ballot(top > m + 8.f) != 0) {
      const float next = top > m ? top : m;
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
        // (a load of 64 tokens holds two steps' rows: half of the lanes write each)
        constexpr bool kHalf = kTok > kWin;
        const int ld = kHalf ? kc * kWin / kTok : kc * kPerWin + k;
        const int tk = kHalf ? lane / kLanes - (kc * kWin) % kTok : lane / kLanes + k * kTok;
        const u32x4 w = vr[ld];
        if (!kHalf || (tk >= 0 && tk < kWin)) {
          const int ln = lane % kLanes;
          if constexpr (kKind <= 1) {
            *(lds_u32x4*)(win + piece_at<kD>(tk, ln)) = w;
          } else {
            constexpr int kOut = kKind == 2 ? 2 : 4;
            const int turn = write_turn<kKind, kD>(tk, ln);
            const uint32_t at = piece_at<kD>(tk, ln * kOut + turn);
            u32x4 out[kOut];
            widen<kBf16, kKind>(
                w, kKind == 3 ? e8m0_scale(exp_s[wave][1][kc * kWin + tk][ln]) : 0.f, turn, out);
#pragma unroll
            for (int y = 0; y < kOut; ++y) *(lds_u32x4*)(win + (at ^ (y << 4))) = out[y];
          }
        }
      }
      order_lds();
      if constexpr (kMore) {
        if (kc == kKC - 1) {   // V is in the window: the next round's loads
          load_rows(vplane, vr);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      // P operand: tokens 4*grp..+3 of tile 2kc, then of tile 2kc+1
      typename Act<kBf16>::x8 w;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int tile = 2 * kc + (j >> 2);
        w[j] = static_cast<Elem>(tile < kTiles ? sc[tile < kTiles ? tile : 0][j & 3] : 0.f);
      }
      // V operand rows: lane 16*grp + rho supplies the row of token 4*grp + rho/4 of the first
      // tile (then of the second), elements 4*(rho%4)..+3 of the 16-element chunk
      // (piece 2 dc + .. of the row at r1 ^ 32 dc; 16 rows on the swizzle is the same)
      const uint32_t r1 = piece_at<kD>(4 * grp + row / 4, row >> 1 & 1) + (row & 1) * 8;
#pragma unroll
      for (int dc = 0; dc < kDC; ++dc) {
        const i16x4 x1 = lds_read_tr16(win + (r1 ^ (dc << 5)));
        i16x4 x2 = {0, 0, 0, 0};
        if constexpr (kTiles > 1) x2 = lds_read_tr16(win + (r1 ^ (dc << 5)) + 16 * kRowV);
        const i16x8 xv = {x1[0], x1[1], x1[2], x1[3], x2[0], x2[1], x2[2], x2[3]};
        o[dc] = mfma16<kBf16>(__builtin_bit_cast(u32x4, xv), __builtin_bit_cast(u32x4, w), o[dc]);
      }
    }
  };
  for (int i = 0; i + 1 < rounds; ++i) round(i, std::true_type{});
  if (rounds > 0) round(rounds - 1, std::false_type{});

  // ---- merge the waves: [m, l] and O[head][d] per wave into LDS
  l = groups_reduce<false>(l);
  if (__ballot(bad) != 0 && rounds > 0) l = __builtin_nanf("");
  __syncthreads();  // the windows are reused for the merge
  float* mrg = reinterpret_cast<float*>(lds);        // [wave][head][kRec]
  if (row < G) {
    float* rec = mrg + (wave * 16 + row) * kRec;
    if (grp == 0) {
      rec[0] = m;
      rec[1] = l;
    }
#pragma unroll
    for (int dc = 0; dc < kDC; ++dc) {
      *reinterpret_cast<f32x4*>(rec + 4 + dc * 16 + 4 * grp) = o[dc];
    }
  }
  __syncthreads();
  for (int i = tid; i < G * (kD / 4); i += kThreads) {
    const int g = i / (kD / 4), d = i % (kD / 4) * 4;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, mrg[(w * 16 + g) * kRec]);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float* wr = mrg + (w * 16 + g) * kRec;
      // (a wave whose scores are all NaN has no maximum, but a sum)
      const float f = wr[0] == -INFINITY ? (wr[1] == 0.f ? 0.f : 1.f)
                                         : __builtin_amdgcn_exp2f(wr[0] - top);
      if (f == 0.f) continue;
      x += *reinterpret_cast<const f32x4*>(wr + 4 + d) * f;
      total += wr[1] * f;
    }
    if (splits == 1) {
      typedef Elem Elem4 __attribute__((ext_vector_type(4)));
      const f32x4 y = x * (total == 0.f ? 0.f : 1.f / total);
      *reinterpret_cast<Elem4*>(reinterpret_cast<Elem*>(a.out) + to + g * kD + d) =
          Elem4{static_cast<Elem>(y.x), static_cast<Elem>(y.y), static_cast<Elem>(y.z),
                static_cast<Elem>(y.w)};
      continue;
    }
    float* rec = a.workspace + (((int64_t)r * H * G + h * G + g) * splits + split) * (kD + 2);
    *reinterpret_cast<f32x4_in*>(rec + 2 + d) = x;
    if (d == 0) *reinterpret_cast<f32x2_in*>(rec) = f32x2{top, total};
  }
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
    const float w = ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f)
                                      : __builtin_amdgcn_exp2f(ml.x - top);
    total += w == 0.f ? 0.f : ml.y * w;
    for (int s = wave; s < 64 && base + s < ns; s += 4 * kCW) {
      float y[4][4], ws[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = s + j * kCW;
        const bool ok = t < 64 && base + t < ns;
        ws[j] = ok ? __shfl(w, t & 63, 64) : 0.f;
        const float* rec = rec0 + (ok ? base + t : base + s) * rs + 2;
#pragma unroll
        for (int c = 0; c < 4; ++c) y[j][c] = c * 64 + lane < D ? rec[c * 64 + lane] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] += ws[j] == 0.f ? 0.f : ws[j] * y[j][c];
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

// Units of 32 KiB of K (at least a round) per split, by the estimate of decode_split_units(): the
// workgroups' rounds through the chip plus half a workgroup's time.
Splits single_splits(const PromptArgs& a, int kind) {
  const int head = head_bytes(kind, a.head_dim);
  const int round = kWaves * wave_tokens(kind, a.head_dim);
  const int64_t unit_tokens = (32768 / head + round - 1) / round * round;
  int64_t most = a.max_tokens;
  if (a.window > 0 && (int64_t)a.window + a.sinks < most) most = (int64_t)a.window + a.sinks;
  const int64_t pairs = (int64_t)a.num_reqs * a.num_kv_heads;
  const int resident = 256 * (a.head_dim > 128 ? 2 : 3);
  const double start = 3.0;
  const double unit = 2.0 * unit_tokens * head * resident / 7e6;   // us
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

template <bool kBf16, int kKind>
auto pick_single(int head_dim) -> void (*)(PromptArgs, int, int) {
  switch (head_dim) {
    case 32: return single_kernel<kBf16, kKind, 32>;
    case 64: return single_kernel<kBf16, kKind, 64>;
    case 128: return single_kernel<kBf16, kKind, 128>;
    case 256: return single_kernel<kBf16, kKind, 256>;
    default: return nullptr;
  }
}

constexpr int kManySplits = 32;   // more: 16 waves merge a row's records, else 4

}  // namespace

int64_t single_workspace_bytes(const PromptArgs& a, int kind) {
  const Splits s = single_splits(a, kind);
  if (s.count == 1) return 0;
  return (int64_t)a.num_reqs * a.num_kv_heads * a.group * s.count * (a.head_dim + 2) * 4;
}

hipError_t launch_single(const PromptArgs& a, bool bf16, int kind, hipStream_t stream) {
  const Splits s = single_splits(a, kind);
  const int64_t groups =
      decode_grid_groups((int64_t)a.num_reqs * decode_grid_splits(s.count)) * a.num_kv_heads;
  const int64_t rows = (int64_t)a.num_reqs * a.num_kv_heads * a.group;
  if (groups > INT32_MAX || rows > INT32_MAX) return hipErrorInvalidValue;
  void (*kernel)(PromptArgs, int, int) = nullptr;
  switch (kind) {
    case 0: kernel = pick_single<false, 0>(a.head_dim); break;
    case 1: kernel = pick_single<true, 1>(a.head_dim); break;
    case 2: kernel = bf16 ? pick_single<true, 2>(a.head_dim) : pick_single<false, 2>(a.head_dim); break;
    case 3: kernel = pick_single<true, 3>(a.head_dim); break;
    default: break;
  }
  if (kernel == nullptr) return hipErrorInvalidValue;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(groups)), dim3(kThreads), 0, stream, a,
                     s.tokens, s.count);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || s.count == 1) return e;
  const bool many = s.count > kManySplits;
  const auto combine = bf16 ? (many ? single_combine<true, 16> : single_combine<true, 4>)
                            : (many ? single_combine<false, 16> : single_combine<false, 4>);
  hipLaunchKernelGGL(combine, dim3(static_cast<unsigned>(rows)), dim3(64 * (many ? 16 : 4)), 0,
                     stream, a, s.tokens, s.count);
  return hipGetLastError();
}

}  // namespace vtoken
