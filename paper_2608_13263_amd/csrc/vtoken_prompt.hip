// Attention of a ragged batch of queries over the paged cache (vtoken_paged_attention): causal,
// with a sliding window and first tokens that stay visible, through a slot mapping.
//
//   prompt_kernel    one workgroup per (tile of query rows, KV head, split): both products on the
//                    matrix cores, a running softmax over 64 keys at a time
//   combine_kernel   merges the splits (no launch where there is one)
//
// A tile's rows are its tokens times the query heads of the KV head, so that one pass over K and V
// serves them all.
//
//   out = sum_k w_k V_k / sum_k w_k,  w_k = 2^(x_k - m),  x_k = q . K_k scale log2(e),
// m a running reference near the row's maximum: where it grows, the sums so far are multiplied by
// 2^(old - new). The partial sums of splits are joined by the same rule.
#include <math.h>

#include "vtoken_elements.h"

namespace vtoken {
namespace {

using namespace elements;

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 32 * kWaves;   // query rows of a tile: (token, query head of the KV head)

// Keys of a step; with 512-byte head rows half as many (registers of the loads in flight, LDS).
constexpr int key_tile(int head_dim) { return head_dim > 128 ? 32 : 64; }

constexpr int kMaxSplits = 64;

// Tokens of a tile.
__host__ __device__ constexpr int tile_tokens(int group) { return kRows / group; }

// A request's part of a call.
struct Request {
  int r;        // -1: no tile of any request
  int q0, ql;   // its queries
  int tile;     // tile of the request
};

// The request that holds tile `tau` of the batch, requests' tiles one after the other. Every lane
// gets the answer; 64 requests at a time.
__device__ __forceinline__ Request find_request(const PromptArgs& a, int tau) {
  Request f{-1, 0, 0, 0};
  const int lane = threadIdx.x & 63;
  const int tq = tile_tokens(a.group);
  const int most = (a.max_queries + tq - 1) / tq;
  for (int base = 0; base < a.num_reqs; base += 64) {
    const int r = base + lane;
    const int q0 = r < a.num_reqs ? a.q_indptr[r] : 0;
    const int q1 = r < a.num_reqs ? a.q_indptr[r + 1] : 0;
    const bool ok = q0 >= 0 && q1 > q0 && q1 <= a.num_queries;
    // (one of more queries than the call allows has the tiles of those that it does: the grid's)
    const int tiles = ok ? min((q1 - q0 + tq - 1) / tq, most) : 0;
    const int incl = meta::wave_inclusive_scan(tiles);
    const uint64_t above = __ballot(incl > tau);
    if (above != 0) {
      const int at = __ffsll(static_cast<long long>(above)) - 1;
      f.r = base + at;
      f.q0 = __builtin_amdgcn_readlane(q0, at);
      f.ql = __builtin_amdgcn_readlane(q1, at) - f.q0;
      // the last tiles of a prompt see the most keys: they go first
      const int first = __builtin_amdgcn_readlane(incl - tiles, at);
      f.tile = __builtin_amdgcn_readlane(tiles, at) - 1 - (tau - first);
      return f;
    }
    tau -= __builtin_amdgcn_readlane(incl, 63);
  }
  return f;
}

// A stored value (not of 4-bit rows).
template <int kKind>
__device__ __forceinline__ float element(const uint8_t* at) {
  if constexpr (kKind == 0) {
    return static_cast<float>(*reinterpret_cast<const _Float16*>(at));
  } else if constexpr (kKind == 1) {
    return static_cast<float>(*reinterpret_cast<const __bf16*>(at));
  } else {
    return __builtin_amdgcn_cvt_f32_fp8(*at, 0);
  }
}

template <bool kBf16>
__device__ __forceinline__ f32x16 mfma32(u32x4 x, u32x4 y, f32x16 acc) {
  if constexpr (kBf16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x),
                                                   __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x),
                                                  __builtin_bit_cast(f16x8, y), acc, 0, 0, 0);
  }
}

// sum + the two elements of pair i of w.
template <bool kBf16>
__device__ __forceinline__ float add_pair(const typename Act<kBf16>::x8& w, int i, float sum) {
  typedef typename Act<kBf16>::x2 X2;
  typedef typename Act<kBf16>::elem Elem;
  const X2 x = {w[2 * i], w[2 * i + 1]}, one = {static_cast<Elem>(1.f), static_cast<Elem>(1.f)};
  if constexpr (kBf16) {
    return __builtin_amdgcn_fdot2_f32_bf16(x, one, sum, false);
  } else {
    return __builtin_amdgcn_fdot2(x, one, sum, false);
  }
}

// x combined with the value of lane i ^ 32.
template <bool kMax>
__device__ __forceinline__ float halves(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const float a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
  return kMax ? fmaxf(a, b) : a + b;
}

// w with the 16-bit halves that are infinities or NaN as zeros.
template <bool kBf16>
__device__ __forceinline__ uint32_t only_finite(uint32_t w) {
  constexpr uint32_t e = kBf16 ? 0x7f80u : 0x7c00u;
  if ((w & e) == e) w &= 0xffff0000u;
  if ((w & e << 16) == e << 16) w &= 0xffffu;
  return w;
}

// 128 rows by 64 keys a step, 32 rows a wave. S^T = K Q^T leaves a lane one row's scores, so that the
// maximum and the sum of a row are a lane's own but for one exchange, and S^T as it comes out is the
// operand of O^T = V^T P^T: no score goes through LDS. K and V of 16 bits go from memory to LDS without
// registers, a step ahead; V is read transposed.
// Weights are rounded to the activations' type for the product, half a step each; the sum is that of the
// rounded ones, and the output is rounded once. In two parts, as single tokens' weights are, they would be
// off by 2^-15 of themselves instead of 2^-8, for 576 us instead of 443 (16 bits), 476 instead of 373
// (8 bits) and 52 instead of 45 (4 bits, few queries of many keys): not taken.
//
// Measured: 8,192 queries with a window of 4,096, 32 query and 8 KV heads of 128, 16 bits, 412.6 GFLOP:
// 443 to 468 us on different cards, 880 to 930 TFLOP/s, three quarters of a large library product's 1,202 to
// 1,215. Counters: matrix cores busy 44% of the time, vector instructions 51%, LDS 23% without conflicts;
// HBM idle. In an earlier version, without the exponentials or with half of the V reads it took 3 to 5%
// less, without the loads 15: none of them was the bound, the order within a wave and the clock under this
// load were.
// Measured and not kept: 64 rows by 32 keys a wave, which halves the reads of LDS (2,048 queries of 4,096
// keys 180 us instead of 138, 26 registers spilled; one workgroup per CU, none spilled, 209; 64 dims 90.5
// instead of 88); scores a step ahead of the weights (16 bits of 128 dims 2 to 7% faster where a request
// has 8,192 keys and no window, the same at the size above; 8 bits 1% and 64 dims 4% slower).
//
// (Two workgroups per CU also at 256 dims, where that spills registers: 4,096 queries of 8,192 keys, 4 KV
// heads with 2 query heads each, take 349 to 355 us instead of 485 in fp8, 308 to 323 instead of 401 in
// 4 bits.)
template <bool kBf16, int kKind, int kD>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(2)))
void prompt_kernel(PromptArgs a) {
  using Elem = typename Act<kBf16>::elem;
  constexpr int kKeys = key_tile(kD);
  constexpr int kTiles = kKeys / 32;        // 32-key score tiles
  constexpr int kChunks = kD / 16;          // score k-steps
  constexpr int kDC = kD / 32;              // 32-element value chunks
  // 16-bit rows go straight to LDS, others through registers, where they are widened
  constexpr bool kDirect = kKind <= 1;
  constexpr int kRow = kD * 2;              // bytes of a row in LDS
  // loads of a step: 16 bytes of a head row each
  constexpr int kLanes = kKind <= 1 ? kD / 8 : kKind == 2 ? kD / 16 : kD / 32;
  constexpr int kItems = kKeys * kLanes;    // of K, and as many of V
  constexpr int kLd = 2 * kItems > kThreads ? 2 * kItems / kThreads : 1;
  constexpr int kSl = kLd > 1 ? kLd / 2 : 1;     // slots of a thread: K and V rows are the same
  // two buffers of K rows, then V rows; two objects, so that a read of one is known not to wait
  // for the loads into the other
  __shared__ __attribute__((aligned(1024))) uint8_t lds0[2 * kKeys * kRow];
  __shared__ __attribute__((aligned(1024))) uint8_t lds1[2 * kKeys * kRow];
  __shared__ int odd_step[2];   // the last step, by buffer, whose V had infinities or NaN

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % a.num_kv_heads;
  const int split = blockIdx.y;
  const Request f = find_request(a, blockIdx.x / a.num_kv_heads);
  if (f.r < 0) return;
  const int G = a.group;
  const int tq = tile_tokens(G);
  const int i0 = f.tile * tq;
  if (f.ql > a.max_queries) {   // its queries are NaN, the last tile's and those past it one after the other
    if (split != 0) return;
    const int end = f.tile == (a.max_queries + tq - 1) / tq - 1 ? f.ql : i0 + tq;
    for (int i = i0; i < end; ++i) {
      Elem* dst = reinterpret_cast<Elem*>(a.out) + (int64_t)(f.q0 + i) * a.out_stride + (int64_t)h * G * kD;
      for (int d = tid; d < G * kD; d += kThreads) dst[d] = static_cast<Elem>(__builtin_nanf(""));
    }
    return;
  }
  const int s0 = a.slot_indptr[f.r];
  const int n = a.slot_count != nullptr ? a.slot_count[f.r] : a.slot_indptr[f.r + 1] - s0;
  const bool fixed = s0 < 0 || n < 0 || n > a.max_tokens;

  // ---- this lane's query row, and the keys that the tile's and the wave's rows see
  const int half = lane >> 5;
  const int m_row = wave * 32 + (lane & 31);
  const int tok = m_row / G;
  const int last = min(i0 + tq, f.ql) - 1;            // last token of the tile
  const bool real = tok < tq && i0 + tok <= last;
  const int rank0 = n - f.ql;                         // rank of the request's query 0
  const int p = real ? rank0 + i0 + tok : -1;
  const int upper = max(rank0 + last + 1, 0);         // keys [0, upper) matter
  const int low = a.window > 0 ? max(rank0 + i0 - a.window + 1, 0) : 0;
  const int sk = min(a.sinks, min(low, upper));       // keys [0, sk) and [low, upper): the list
  const int skip = low - sk;
  const int count = fixed ? 0 : sk + max(upper - low, 0);
  const int steps = (count + kKeys - 1) / kKeys;
  const int step0 = static_cast<int>((int64_t)steps * split / gridDim.y);
  const int step1 = static_cast<int>((int64_t)steps * (split + 1) / gridDim.y);
  const int w_tok0 = i0 + wave * 32 / G;
  const int w_first = rank0 + w_tok0;                                        // ranks of the wave's
  const int w_last = rank0 + min(i0 + (wave * 32 + 31) / G, last);           // first and last row
  const bool w_real = w_tok0 <= last && wave * 32 < tq * G;

  // ---- the query operand: element e of chunk c is value 16 c + 8 half + e of the row
  u32x4 q[kChunks];
  {
    // (a row past the tile takes another's query; its results are not written)
    const Elem* src = reinterpret_cast<const Elem*>(a.q) +
                      (int64_t)(f.q0 + min(i0 + tok, last)) * a.q_stride +
                      (int64_t)(h * G + (real ? m_row - tok * G : 0)) * kD + 8 * half;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      q[c] = *reinterpret_cast<const u32x4*>(src + 16 * c);
      if (a.scale < 0.f) q[c] ^= 0x80008000u;
      if (a.scale == 0.f) q[c] = u32x4{0, 0, 0, 0};
    }
  }
  // weights are powers of two, with a positive factor (a hidden key's -inf stays one)
  const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.44269504088896340736f;

  // ---- loads
  const uint32_t num_slots = static_cast<uint32_t>(a.num_slots);
  const uint8_t* kplane = a.kv + (int64_t)(2 * a.layer) * a.plane_bytes;
  // slots of a step's rows; those past the list re-read its last one
  const int32_t* slots = a.slots + s0;
  auto load_slots = [&](int j, uint32_t (&s)[kSl]) {
#pragma unroll
    for (int x = 0; x < kSl; ++x) {
      const int t = min(j * kKeys + (tid + x * kThreads) / kLanes % kKeys, count - 1);
      s[x] = static_cast<uint32_t>(slots[t + (t < sk ? 0 : skip)]);
    }
  };
  // whether one of them is outside the pool
  auto any_outside = [&](const uint32_t (&s)[kSl]) {
    uint32_t most = 0;
#pragma unroll
    for (int x = 0; x < kSl; ++x) most = max(most, s[x]);
    return __ballot(most >= num_slots) != 0;
  };
  u32x4 data[kDirect ? 1 : kLd];
  uint32_t exponent[kKind == 3 ? kLd : 1];
  const uint32_t row_bytes = static_cast<uint32_t>(a.row_bytes);
  auto load_row = [&](int x, const uint32_t (&s)[kSl], lds_u8* buf) {   // item x of this thread's
    const int item = tid + x * kThreads;
    if (2 * kItems < kThreads && item >= 2 * kItems) return;
    const bool is_v = kLd > 1 ? x >= kLd / 2 : item >= kItems;
    const uint32_t slot = s[x % kSl] < num_slots ? s[x % kSl] : 0u;
    const int ln = item % kLanes;
    const uint8_t* plane = is_v ? kplane + a.plane_bytes : kplane;
    if constexpr (kDirect) {
      // a wave's 64 pieces follow each other in LDS: the lane picks the piece that belongs there
      const uint8_t* src = plane +
                           (h * kLanes + (ln ^ swizzle<kD>(item / kLanes % kKeys))) * 16 +
                           (uint64_t)slot * row_bytes;
      typedef __attribute__((address_space(1))) const uint32_t global_u32;
      typedef __attribute__((address_space(3))) uint32_t lds_u32;
      __builtin_amdgcn_global_load_lds(
          (global_u32*)(reinterpret_cast<uintptr_t>(src)),
          (lds_u32*)(buf + (wave * 64 + x * kThreads) * 16), 16, 0, 0);
    } else {
      const uint8_t* row = plane + (uint64_t)slot * row_bytes;
      data[x] = *reinterpret_cast<const u32x4*>(row + (h * kLanes + ln) * 16);
      if constexpr (kKind == 3) {
        exponent[x] = row[a.num_kv_heads * (kD / 2) + h * (kD / 32) + ln];
      }
    }
  };
  auto load_rows = [&](const uint32_t (&s)[kSl], lds_u8* buf) {
#pragma unroll
    for (int x = 0; x < kLd; ++x) load_row(x, s, buf);
  };
  // What step j's rows still need before they can be read: the widened values; where a row is past
  // the list (V: zeros, K: anything) or outside the pool (V: zeros, K: NaN); and where some row does
  // not see all keys (`look`), zeros for V's infinities and NaN, since a zero weight times one of
  // them would be NaN.
  auto stage = [&](int j, const uint32_t (&s)[kSl], lds_u8* buf, bool look) {
    if constexpr (kDirect) {
      __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): this wave's pieces are in LDS
      if (!look) return;                    // (the list's end is a step of that kind)
    }
    bool odd = false;
    // piece y of item x is at (at ^ 16 y) + the rows of x items, formed anew in each step
    constexpr int kOut = kKind <= 1 ? 1 : kKind == 2 ? 2 : 4;   // 16-byte pieces of LDS
    constexpr int kPass = kThreads / kLanes;                    // rows of an item of every thread
    static_assert(kDirect || kPass % 16 == 0, "the items' rows have one swizzle");
    int thread = tid;
    asm volatile("" : "+v"(thread));
    const int turn = write_turn<kKind, kD>(thread / kLanes % kKeys, thread % kLanes);
    const uint32_t at = piece_at<kD>(thread / kLanes % kKeys, thread % kLanes * kOut + turn);
#pragma unroll
    for (int x = 0; x < kLd; ++x) {
      const int item = thread + x * kThreads;
      if (2 * kItems < kThreads && item >= 2 * kItems) break;
      const bool is_v = kLd > 1 ? x >= kLd / 2 : item >= kItems;
      lds_u8* dst = buf + (is_v ? kKeys * kRow : 0);
      u32x4 o[kOut];
      if constexpr (kDirect) {
        dst += piece_at<kD>(item / kLanes % kKeys, item % kLanes ^ swizzle<kD>(item / kLanes % kKeys));
        o[0] = *(lds_u32x4*)dst;
      } else {
        widen<kBf16, kKind>(data[x], kKind == 3 ? e8m0_scale(exponent[kKind == 3 ? x : 0]) : 0.f,
                            turn, o);
      }
      // (all of this is put right by every step that may need it, `look`)
      const bool past = look && j * kKeys + item / kLanes % kKeys >= count;
      const bool outside = look && s[x % kSl] >= num_slots;
      if (past || outside) {
        const uint32_t fill = past || is_v ? 0u : 0x7fff7fffu;
#pragma unroll
        for (int y = 0; y < kOut; ++y) o[y] = u32x4{fill, fill, fill, fill};
      }
      if (kKind == 3 && look && is_v) {   // (6 x 2^125 is bf16's last; the codes are finite)
        if (exponent[kKind == 3 ? x : 0] > 252) {
          odd |= !past && !outside;
#pragma unroll
          for (int y = 0; y < kOut; ++y) o[y] = u32x4{0, 0, 0, 0};
        }
      } else if (look && is_v) {
#pragma unroll
        for (int y = 0; y < kOut; ++y)
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const uint32_t w = only_finite<kBf16>(o[y][z]);
            odd |= w != o[y][z];
            o[y][z] = w;
          }
      }
#pragma unroll
      for (int y = 0; y < kOut; ++y) {
        if constexpr (kDirect) {
          *(lds_u32x4*)dst = o[y];
        } else {
          *(lds_u32x4*)(dst + (at ^ (y << 4)) + x % kSl * (kPass * kRow)) = o[y];
        }
      }
    }
    if (look && odd) odd_step[j & 1] = j;
  };
  // whether every key of step j is seen by all of the rows of ranks [first, last]
  auto all_seen = [&](int j, int first, int lst) {
    const int t0 = j * kKeys, t1 = t0 + kKeys - 1;
    const int kmin = t0 + (t0 < sk ? 0 : skip), kmax = t1 + (t1 < sk ? 0 : skip);
    return t1 < count && kmax <= first &&
           (a.window == 0 || kmax < a.sinks || (t0 >= sk && kmin > lst - a.window));
  };

  const int hidden = a.window > 0 ? p - a.window : INT32_MIN;   // the last key before the window
  auto seen = [&](int k) { return (k <= p) & ((k > hidden) | (k < a.sinks)); };

  float m = -INFINITY, l = 0.f;
  f32x16 o[kDC];
#pragma unroll
  for (int dc = 0; dc < kDC; ++dc)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dc][e] = 0.f;

  uint32_t sa[kSl], sb[kSl];   // slots of this step and, when its rows are asked for, the next
  // One step of the wave's rows. The next step's rows that go straight to `other` are asked for beside the
  // first of its value products, one each: all at once, after the barrier, the waves wait for each other's
  // (4 x 1,024 queries of 8,192 keys of 16 bits 526 us instead of 572; rows that go through registers
  // 1 to 2% slower that way).
  auto compute = [&](int j, const lds_u8* buf, lds_u8* other) {
    // K piece 2 c + half of row lane & 31 is at at_k ^ 32 c; V piece 4 dc + vpiece of row vrow at
    // at_v ^ 64 dc, of row vrow + 8 at (at_v ^ 64 dc ^ 16) + 8 rows: formed anew in each step (kept
    // over the loop they would take two dozen registers)
    uint32_t at_k = piece_at<kD>(lane & 31, half);
    uint32_t at_v = piece_at<kD>(4 * half + (lane & 15) / 4,
                                 (lane >> 4 & 1) * 2 + (lane >> 1 & 1)) + (lane & 1) * 8;
    asm volatile("" : "+v"(at_k), "+v"(at_v));
    // ---- scores: lane holds keys 32 t + 8 (i / 4) + 4 half + i % 4 of its row
    f32x16 s[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const lds_u8* src = buf + (at_k ^ (c << 5)) + 32 * t * kRow;
        s[t] = mfma32<kBf16>(*(const lds_u32x4*)src, q[c], s[t]);
      }
    // reads four products ahead
    constexpr int kAhead = kChunks * kTiles < 4 ? kChunks * kTiles : 4;
    __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
    for (int x = 0; x < kChunks * kTiles - kAhead; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
    auto key_of = [&](int t, int e) {   // rank of the lane's key, or past every row's
      const int x = j * kKeys + 32 * t + 8 * (e / 4) + 4 * half + e % 4;
      const int k = x + (x < sk ? 0 : skip);
      return x >= count ? INT32_MAX : k;
    };
    if (!all_seen(j, w_first, w_last)) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[t][e] = seen(key_of(t, e)) ? s[t][e] : -INFINITY;
        }
    }
    // ---- weights 2^(x - m), see Act
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[t][e]);
    top = halves<true>(top) * scale;
    if (__ballot(top > m + Act<kBf16>::kMost) != 0) {
      const float to = fmaxf(top - Act<kBf16>::kFirst, m);
      const float by = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= by;
#pragma unroll
      for (int dc = 0; dc < kDC; ++dc)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dc][e] *= by;
    }
    const float base = m == -INFINITY ? 0.f : m;
    // ---- O^T += V^T . P^T, 16 keys at a time: a lane's weights 8 y .. 8 y + 7 of tile t are keys
    // 16 y + 4 half + (0..3) and those eight on; the V rows are read in that order. The weights of
    // the next 16 keys are formed while the matrix cores work on these.
    const lds_u8* vbuf = buf + kKeys * kRow;
    constexpr int kGroups = 2 * kTiles;       // of 16 keys
    constexpr int kPart = 8 / kDC > 0 ? 8 / kDC : 1;   // weights formed beside a product
    auto weights = [&](typename Act<kBf16>::x8& w, int g, int e0, int n) {
#pragma unroll
      for (int e = e0; e < e0 + n && e < 8; ++e) {
        w[e] = static_cast<Elem>(__builtin_amdgcn_exp2f(
            __builtin_fmaf(s[g / 2][8 * (g % 2) + e], scale, -base)));
        // the sum is that of the rounded weights, which the product takes
        if (e % 2 == 1) l = add_pair<kBf16>(w, e / 2, l);
      }
    };
    auto v_operand = [&](int x) {   // of product x: group x / kDC, values 32 (x % kDC) ..
      const lds_u8* src = vbuf + 16 * (x / kDC) * kRow;
      const int dc = x % kDC;
      const i16x4 x1 = lds_read_tr16(src + (at_v ^ (dc << 6)));
      const i16x4 x2 = lds_read_tr16(src + (at_v ^ (dc << 6 | 16)) + 8 * kRow);
      const i16x8 v = {x1[0], x1[1], x1[2], x1[3], x2[0], x2[1], x2[2], x2[3]};
      return __builtin_bit_cast(u32x4, v);
    };
    __builtin_amdgcn_s_setprio(1);
    // (a wave in its value products goes first: 4 x 1,024 queries of 8,192 keys in 8 bits 532 us; with that
    // for its scores 559; 16 bits and 128 dims take the same)
    constexpr int kProducts = kGroups * kDC;
    static_assert(!kDirect || kLd <= kProducts, "a load beside a product");
    u32x4 v[3] = {v_operand(0), v_operand(1 < kProducts ? 1 : 0), {}};
    typename Act<kBf16>::x8 w[2];
    weights(w[0], 0, 0, 8);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int x = 0; x < kProducts; ++x) {
      const int g = x / kDC, dc = x % kDC;
      if (x + 2 < kProducts) v[(x + 2) % 3] = v_operand(x + 2);
      o[dc] = mfma32<kBf16>(v[x % 3], __builtin_bit_cast(u32x4, w[g & 1]), o[dc]);
      if (g + 1 < kGroups) weights(w[(g + 1) & 1], g + 1, dc * kPart, kPart);
      if (kDirect && x < kLd) load_row(x, sa, other);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  };
  // Step j's infinities and NaN of V, which LDS holds as zeros, for the rows that see them (from the
  // cache: this is rare, and a row that sees one is lost anyway)
  auto add_nonfinite = [&](int j) {
#pragma unroll 1
    for (int t = j * kKeys; t < min((j + 1) * kKeys, count); ++t) {
      const int k = t + (t < sk ? 0 : skip);
      const int slot = a.slots[(int64_t)s0 + k];
      if (static_cast<unsigned>(slot) >= static_cast<unsigned>(a.num_slots) || !seen(k)) continue;
      const uint8_t* row = kplane + a.plane_bytes + (int64_t)slot * a.row_bytes;
#pragma unroll
      for (int dc = 0; dc < kDC; ++dc)
        if constexpr (kKind == 3) {   // an exponent's 32 values are lost, or none
          if (row[a.num_kv_heads * (kD / 2) + h * (kD / 32) + dc] <= 252) continue;
#pragma unroll
          for (int e = 0; e < 16; ++e) o[dc][e] = __builtin_nanf("");
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float v =
                element<kKind>(row + (h * kD + 32 * dc + 8 * (e / 4) + 4 * half + e % 4) *
                                         (kKind <= 1 ? 2 : 1));
            if (!(fabsf(v) < INFINITY)) o[dc][e] += v;
            // (with all loads at once their registers cost a prompt of 128 dims 485 us instead of 460)
            if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
          }
        }
    }
  };

  // Step j from `buf`, the next step's rows on their way to `other`. One barrier a step: `other`
  // was last read in step j - 1, which every wave has left when it passes step j's barrier.
  lds_u8* const buf0 = (lds_u8*)lds0;
  lds_u8* const buf1 = (lds_u8*)lds1;
  auto step = [&](int j, lds_u8* buf, lds_u8* other) {
    // (also where a slot may be outside the pool: those are looked for in every step)
    const bool look = !all_seen(j, rank0 + i0, rank0 + last) || any_outside(sa);
    stage(j, sa, buf, look);
    const bool more = j + 1 < step1;
    if (!kDirect && more) load_rows(sb, other);
    __syncthreads();
    const int k0 = j * kKeys + (j * kKeys < sk ? 0 : skip);
    const bool none = !w_real || k0 > w_last;
    if (kDirect && none && more) load_rows(sb, other);
#pragma unroll
    for (int x = 0; x < kSl; ++x) sa[x] = sb[x];
    if (j + 2 < step1) load_slots(j + 2, sb);
    if (none) return;
    compute(j, buf, other);
    if (odd_step[j & 1] == j) add_nonfinite(j);
  };
  if (tid < 2) odd_step[tid] = -1;
  if (step0 < step1) {
    load_slots(step0, sa);
    load_rows(sa, buf0);
    load_slots(step0 + 1, sb);
  }
  __syncthreads();   // odd_step
  for (int j = step0; j < step1; j += 2) {
    step(j, buf0, buf1);
    if (j + 1 < step1) step(j + 1, buf1, buf0);
  }
  // the last step's loads, which nothing reads, must not outlive the workgroup's LDS
  if constexpr (kDirect) __builtin_amdgcn_s_waitcnt(0x0f70);

  // ---- the rows' results: lane holds values 32 dc + 8 (e / 4) + 4 half + e % 4
  int at_row = m_row;   // (the row's place is worked out again, not kept over the loop)
  asm volatile("" : "+v"(at_row));
  const int tok2 = at_row / G;
  if (tok2 >= tq || i0 + tok2 > last) return;
  const int64_t qrow = f.q0 + i0 + tok2;
  const int qh = h * G + at_row - tok2 * G;
  l = halves<false>(l);
  // what only the epilogue needs is read again, from the kernel's argument
  auto* late = (const __attribute__((address_space(4))) PromptArgs*)
      __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(late));
  if (gridDim.y == 1) {
    const float inv = fixed ? __builtin_nanf("") : l == 0.f ? 0.f : 1.f / l;
    Elem* dst =
        reinterpret_cast<Elem*>(late->out) + qrow * late->out_stride + (int64_t)qh * kD + 4 * half;
    typedef Elem Elem4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int dc = 0; dc < kDC; ++dc)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const Elem4 w = {static_cast<Elem>(o[dc][4 * e] * inv),
                         static_cast<Elem>(o[dc][4 * e + 1] * inv),
                         static_cast<Elem>(o[dc][4 * e + 2] * inv),
                         static_cast<Elem>(o[dc][4 * e + 3] * inv)};
        *reinterpret_cast<Elem4*>(dst + 32 * dc + 8 * e) = w;
      }
    return;
  }
  float* rec = late->workspace +
               ((qrow * late->num_kv_heads * G + qh) * gridDim.y + split) * (kD + 2);
  if (half == 0) {
    rec[0] = fixed ? __builtin_nanf("") : m;
    rec[1] = l;
  }
#pragma unroll
  for (int dc = 0; dc < kDC; ++dc)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<f32x4_in*>(rec + 2 + 32 * dc + 8 * e + 4 * half) =
          f32x4{o[dc][4 * e], o[dc][4 * e + 1], o[dc][4 * e + 2], o[dc][4 * e + 3]};
}

// Merges the split records (m, l, O) of a tile's rows, a row per wave: weights 2^(m_s - max m).
// Bound: latency; every wave reads all the (m_s, l_s) at once and eight records at a time. 768 rows of
// 64 records of 128 dims: 10.5 us (25.6 MB, 2.4 TB/s); a workgroup with its rows one after another took 128.
template <bool kBf16>
__global__ __launch_bounds__(kThreads) void combine_kernel(PromptArgs a, int splits) {
  using Elem = typename Act<kBf16>::elem;
  typedef Elem Elem2 __attribute__((ext_vector_type(2)));
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % a.num_kv_heads;
  const Request f = find_request(a, blockIdx.x / a.num_kv_heads);
  if (f.r < 0 || f.ql > a.max_queries) return;   // (the latter's have been written)
  const int G = a.group, D = a.head_dim;
  const int tq = tile_tokens(G);
  const int tokens = min(tq, f.ql - f.tile * tq);
  const int row = blockIdx.y * kWaves + wave;
  if (row >= tokens * G) return;
  const int64_t qrow = f.q0 + f.tile * tq + row / G;
  const int qh = h * G + row % G;
  const int64_t rs = D + 2;
  const float* rec = a.workspace + (qrow * a.num_kv_heads * G + qh) * splits * rs;
  const f32x2 ml = lane < splits ? *reinterpret_cast<const f32x2_in*>(rec + lane * rs)
                                 : f32x2{-INFINITY, 0.f};
  const bool nan = __ballot(ml.x != ml.x) != 0;
  float top = ml.x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  // (no split is left out: a NaN or an infinity in the sums of one far below the others has to reach
  // the row, also times zero; one without a maximum holds zeros, or NaN)
  const float w = ml.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml.x - top);
  float total = ml.y * w;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d, 64);
  const int p0 = 2 * lane, p1 = 128 + 2 * lane;   // this lane's pairs of values
  f32x2 v0 = {0.f, 0.f}, v1 = {0.f, 0.f};
  for (int s = 0; s < splits; s += 8) {
    f32x2 x0[8], x1[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool ok = s + j < splits;
      const float* src = rec + (ok ? s + j : s) * rs + 2;
      x0[j] = ok && p0 < D ? *reinterpret_cast<const f32x2_in*>(src + p0) : f32x2{0.f, 0.f};
      x1[j] = ok && p1 < D ? *reinterpret_cast<const f32x2_in*>(src + p1) : f32x2{0.f, 0.f};
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float ws = __shfl(w, (s + j) & 63, 64);
      v0 += x0[j] * ws;
      v1 += x1[j] * ws;
    }
  }
  const float inv = nan ? __builtin_nanf("") : total == 0.f ? 0.f : 1.f / total;
  Elem* dst = reinterpret_cast<Elem*>(a.out) + qrow * a.out_stride + (int64_t)qh * D;
  if (p0 < D) {
    *reinterpret_cast<Elem2*>(dst + p0) =
        Elem2{static_cast<Elem>(v0.x * inv), static_cast<Elem>(v0.y * inv)};
  }
  if (p1 < D) {
    *reinterpret_cast<Elem2*>(dst + p1) =
        Elem2{static_cast<Elem>(v1.x * inv), static_cast<Elem>(v1.y * inv)};
  }
}

// Tiles of query rows that a batch can have.
int64_t most_tiles(const PromptArgs& a) {
  const int tq = tile_tokens(a.group);
  const int64_t by_rows = a.num_queries / tq + (int64_t)a.num_reqs;
  const int64_t by_reqs = (int64_t)a.num_reqs * ((a.max_queries + tq - 1) / tq);
  return by_rows < by_reqs ? by_rows : by_reqs;
}

// Splits fill the chip, two workgroups per CU, where the tiles do not: half as many cost more where the
// keys are many (16 queries of 32,768 keys 55 us instead of 48, 4 x 64 of 8,192 93 instead of 71), more
// than that run one after another (4 x 64 of 8,192: 86 us with 768). A split of fewer than eight steps
// costs more to merge than it saves (512 queries of 512 keys: 31 us at four steps or more, 23 at eight);
// sixteen leave too few (128 queries of 4,096 keys 44 us instead of 32). (Measured before the kernel's last
// steps: as kept, the sizes of one request take 44, 20 and 28 us now.)
int prompt_splits(const PromptArgs& a) {
  const int64_t groups = most_tiles(a) * a.num_kv_heads;
  if (groups == 0) return 1;
  int64_t keys = a.max_tokens;
  if (a.window > 0) {
    const int64_t list = (int64_t)a.window + a.sinks + tile_tokens(a.group);
    keys = list < keys ? list : keys;
  }
  const int64_t steps = (keys + key_tile(a.head_dim) - 1) / key_tile(a.head_dim);
  const int64_t want = (512 + groups - 1) / groups;      // workgroups: two per CU
  int64_t splits = want < steps / 8 ? want : steps / 8;
  if (splits > kMaxSplits) splits = kMaxSplits;
  return splits < 1 ? 1 : static_cast<int>(splits);
}

template <bool kBf16, int kKind>
auto pick_prompt(int head_dim) -> void (*)(PromptArgs) {
  switch (head_dim) {
    case 32: return prompt_kernel<kBf16, kKind, 32>;
    case 64: return prompt_kernel<kBf16, kKind, 64>;
    case 128: return prompt_kernel<kBf16, kKind, 128>;
    case 256: return prompt_kernel<kBf16, kKind, 256>;
    default: return nullptr;
  }
}

}  // namespace

int64_t prompt_workspace_bytes(const PromptArgs& a) {
  const int splits = prompt_splits(a);
  if (splits == 1) return 0;
  return (int64_t)a.num_queries * a.num_kv_heads * a.group * splits * (a.head_dim + 2) * 4;
}

hipError_t launch_prompt(const PromptArgs& a, bool bf16, int kind, hipStream_t stream) {
  const int64_t groups = most_tiles(a) * a.num_kv_heads;
  if (groups > UINT32_MAX / kThreads) return hipErrorInvalidValue;   // (a grid's threads)
  void (*kernel)(PromptArgs) = nullptr;
  switch (kind) {
    case 0: kernel = pick_prompt<false, 0>(a.head_dim); break;
    case 1: kernel = pick_prompt<true, 1>(a.head_dim); break;
    case 2: kernel = bf16 ? pick_prompt<true, 2>(a.head_dim) : pick_prompt<false, 2>(a.head_dim); break;
    case 3: kernel = pick_prompt<true, 3>(a.head_dim); break;
    default: break;
  }
  if (kernel == nullptr) return hipErrorInvalidValue;
  const int splits = prompt_splits(a);
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(groups), splits), dim3(kThreads), 0, stream,
                     a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  const int64_t rows = (int64_t)a.max_queries * a.group;
  const unsigned parts = ((rows < kRows ? static_cast<unsigned>(rows) : kRows) + kWaves - 1) / kWaves;
  hipLaunchKernelGGL(bf16 ? combine_kernel<true> : combine_kernel<false>,
                     dim3(static_cast<unsigned>(groups), parts), dim3(kThreads), 0, stream, a,
                     splits);
  return hipGetLastError();
}

}  // namespace vtoken
