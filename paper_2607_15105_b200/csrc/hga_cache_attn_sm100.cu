// hga_cache_attn for chunks of new tokens (tcgen05 / TMEM / TMA).
//
// A unit is up to 256 query rows of one (sequence, key/value head) -- new tokens x query heads of the group, token by token -- as two
// M-tiles of 128 rows.  Keys come in tiles of 128, which both M-tiles read from one ring in shared memory, and are taken 64 at a time:
// S = Q K^T, P = 2^(S c - m), O += P V, with S, P and O in tensor memory.  An M-tile has two buffers of 64 columns for S, over which
// P is written: while its softmax threads (four warps, a thread per row) work on one, the tensor pipe fills the other, so they find
// the next S ready.  (Steps of 128 keys with one buffer per M-tile, the M-tiles taking turns: 4200 cycles for 2 x 128 x 128, most of them
// waiting for one another.)  Of S's GEMMs, N = 64 costs 1.5 times the cycles per key of N = 128: they are bound by reading Q.
//
//   warps 0-3, 4-7   softmax and epilogue of M-tile 0 and 1
//   warps 8, 9       issue the GEMMs of M-tile 0 and 1
//   warps 10, 11     copy K and V tiles by TMA, a box per page part (quantised pages: as they are, and their scales); e4m3: clean the last V tiles
//   warps 12-15      bf16 pages: clean the last V tiles; quantised: convert K and V tiles
//
// Quantised pages are multiplied as fp16, into which the converter instructions go and which holds e4m3 and e2m1 with their scales
// exactly while these lie in a range of 2^22 (e4m3; Q is brought to fp16 by a power of two per row, exactly but for numbers 2^-29 of
// the row's largest).  A unit that meets another scale starts again in bf16, when it has come to its end: one block of values below 8e-4 in a
// history is enough (12 packed sequences, e4m3, with one each: 541 us -> 1353).
//
// A hidden key has weight zero, which does not silence a V row that is not finite.  So in the tiles that hold keys hidden from the
// unit's first row (the last ones), numbers that are not finite are replaced by zeros, rows behind the last key altogether, and the
// rows that do see such numbers get them added at the end.  (Of quantised pages: blocks with a scale of 255, and e4m3's NaN codes.)
//
// Measured, 32 query heads on 8 of 128, calls one after another: 2048 tokens behind 14336, bf16, 534 to 545 us (0.95 PFLOP/s; tensor pipe active
// 71 % of the time, 256 units on 148 SMs); 16384 tokens 2159 to 2205 us (1.0 PFLOP/s, at the power limit); e4m3, 12 packed sequences 541 to
// 570 us (0.81 to 0.85 PFLOP/s: the shared-memory pipe, 76 to 85 % busy with converted tiles and the GEMMs' operands), e2m1 509.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "hga_cache.cuh"
#include "hga_sm100.cuh"

namespace hga {

using namespace sm100;

namespace {

constexpr int kThreads = 512;
// Registers of a thread of the softmax warps, of GEMMs and copies, of the rest; the launch has 128 for each.
constexpr int kSoftmaxRegs = 184, kIssueRegs = 48, kRestRegs = 96;
static_assert(2 * kSoftmaxRegs + kIssueRegs + kRestRegs <= 4 * 128, "registers of the block");
constexpr int kFill = 4;                   // warps that convert or clean
constexpr int kTile = 128;                 // rows of an M-tile, keys of a tile
constexpr int kStep = 64;                  // keys of a step
constexpr uint32_t kTmemCols = 512;
constexpr float kNoRef = -3e38f;           // reference of a row that has seen no key: 2^(-inf - it) = 0, and any logit raises it
// A row's reference is raised, and O rescaled, when a logit exceeds it by kSlack (log2), to kLow below the row's largest: most tiles
// leave O alone, and fp16 weights go down to 2^-31 of the reference's.
constexpr float kLow = 6.f, kSlack = 14.f;

template <int FMT, int D>
struct Smem {
  static constexpr bool kScaled = FMT != kCacheBf16;
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kSlots = (kScaled ? 4 : 5) * 128 / D;
  static constexpr int kRaw = kScaled ? kTile * cache_row_bytes(FMT, D) : 0, kRawScales = kScaled ? kTile * (D / 32) : 0;
  uint8_t q[2][kTileBytes];                // [panel of 64 elements][row][128 bytes], 128-byte swizzle, as all tiles
  uint8_t ring[kSlots][kTileBytes];        // K and V tiles in turn
  uint8_t raw[2][kScaled ? kRaw + kRawScales : 128];      // quantised tiles as they lie in their pages, rows one behind the other, and their scales
  uint64_t full[kSlots], empty[kSlots];    // full: one arrival of each of the filling warps (four for the copying ones)
  uint64_t raw_full[kSlots];               // K or V to be converted is there (0, 1), e4m3 V to be cleaned first (2); bf16 V to be cleaned (any slot)
  uint64_t raw_empty[2];
  // s_full, p_full: of M-tile x's buffer b.  s_full for the t-th time: S of step 2 t + b is there, if there is such a step, and P V of
  // step 2 t + b - 2 done.
  uint64_t s_full[2][2], p_full[2][2], drain[2];
  // (no member between the barriers)
  int8_t q_up[2 * kTile];                  // fp16: the power of two that a row of Q was multiplied by
  uint32_t tmem_base;
  int abort, strange, wide;                // wide: a scale outside fp16's range
  int seq, token0;                         // the unit's sequence, and its first token there
};

__device__ __align__(16) const uint8_t kNoScales[kTile * 4] = {};      // of keys that are none

constexpr int kMaxRanked = kThreads;       // units, and sequences

struct Plan {
  int tokens;                              // of an M-tile
  int units;                               // per key/value head and part, at most
  bool ranked;                             // by their steps
  int box;                                 // tokens of a TMA box: the largest power of two that divides the page (128 at most)
  Div by_unit;                             // tokens of a unit
  CacheSplit sp;
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// byte offset of 16-byte piece `c` of row r in a tile
template <int D> __device__ __forceinline__ int piece(int r, int c) { return (c >> 3) * (kTile * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4); }

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ bool all_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort));
}

// 2^x of two numbers x < 128 on the FMA pipe, for a share of the weights: the special-function units take 8 cycles per warp and number, which
// bounds the softmax.  x = n + f, |f| <= 1/2, n by adding and subtracting 1.5 2^23; 2^f by a polynomial fitted here for least relative error
// (2.6e-6; weights are rounded to 2^-9 or 2^-12); 2^n from its bits.  Below -127, and for -inf: 0.  NaN stays NaN.
__device__ __forceinline__ void exp2_by_fma(float& x0, float& x1) {
  asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x0));
  asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x1));
  const uint64_t x = pack_f32x2(x0, x1), t = add_f32x2(x, pack_f32x2(12582912.f, 12582912.f));
  const uint64_t n = add_f32x2(t, pack_f32x2(-12582912.f, -12582912.f)), f = fma_f32x2(n, pack_f32x2(-1.f, -1.f), x);
  uint64_t p = pack_f32x2(0.009570101276040077f, 0.009570101276040077f);
  p = fma_f32x2(p, f, pack_f32x2(0.05591785907745361f, 0.05591785907745361f));
  p = fma_f32x2(p, f, pack_f32x2(0.240247443318367f, 0.240247443318367f));
  p = fma_f32x2(p, f, pack_f32x2(0.6931217908859253f, 0.6931217908859253f));
  p = fma_f32x2(p, f, pack_f32x2(0.9999992847442627f, 0.9999992847442627f));
  float t0, t1;
  unpack_f32x2(t, t0, t1);
  p = mul_f32x2(p, pack_f32x2(__uint_as_float((__float_as_uint(t0) << 23) + 0x3f800000u), __uint_as_float((__float_as_uint(t1) << 23) + 0x3f800000u)));
  unpack_f32x2(p, x0, x1);
}

__device__ __forceinline__ bool not_finite(uint32_t bf16_bits) { return (bf16_bits & 0x7f80u) == 0x7f80u; }

template <int FMT, int D>
__global__ void __launch_bounds__(kThreads, 1)
k_cache_attn_sm100(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const CacheDims dm, const Plan plan, const uint16_t* Q, const int32_t* cu_q,
                   const int32_t* seq_lens, const int32_t* table, const uint8_t* K,
                   const uint8_t* V, const uint8_t* K_scale, const uint8_t* V_scale,
                   uint16_t* O, float* LSE, float* part_o, int32_t* status_word) {
  typedef Smem<FMT, D> Sm;
  constexpr int NS = Sm::kSlots;
  extern __shared__ uint8_t raw[];
  Sm& sm = *reinterpret_cast<Sm*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort = &sm.abort;

  if ((warp == 10 || warp == 11) && lane == 0) prefetch_tensormap(warp == 11 ? &map_v : &map_k);
  pdl_wait();
  // Which unit: the longest first, so that the SMs end at one time, and the heads of a unit one after another.  Units are counted off
  // sequence after sequence, and the late tokens of a sequence see most keys; with several sequences they are ranked by their steps
  // (up to 512; 12 sequences of up to 1000 new tokens, 108 units: 633 us in the order of the sequences, 564 so).
  int at = blockIdx.x, part = 0;
  const bool split = plan.sp.parts > 1 && at >= plan.sp.full;
  if (split) {
    // (the first parts, which may be the longer ones, first)
    const int i = at - plan.sp.full, n = plan.units * dm.Hkv - plan.sp.full;
    part = i / n;
    at = plan.sp.full + i - part * n;
  }
  const int rank = dm.by_Hkv(at), h = at - rank * dm.Hkv;
  if (plan.ranked) {
    int* const first = reinterpret_cast<int*>(sm.ring);        // [n_seq + 1] first unit of a sequence
    int* const steps = first + kMaxRanked + 32;                // of a unit
    int* const sums = steps + kMaxRanked;                      // of a warp's sequences
    const int unit = 2 * plan.tokens;
    int n = 0;
    if (tid < dm.n_seq) {
      const CacheSeq s = cache_seq(dm, cu_q, seq_lens, tid);
      n = plan.by_unit(s.n + unit - 1);
      if (s.bad && blockIdx.x == 0) cache_status(status_word, HGA_STATUS_BAD_INDEX);
    }
    int upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) sums[warp] = upto;
    if (tid == 0) sm.seq = -1;
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto += sums[w];
    if (tid < dm.n_seq) first[tid + 1] = upto;
    if (tid == 0) first[0] = 0;
    __syncthreads();
    const int units = min(first[dm.n_seq], kMaxRanked);
    int seq = 0, t0 = 0, mine = 0;
    if (tid < units) {
      int hi = dm.n_seq;                                       // (first[seq] <= tid < first[hi])
      while (hi - seq > 1) {
        const int mid = (seq + hi) >> 1;
        if (first[mid] <= tid) seq = mid; else hi = mid;
      }
      t0 = (tid - first[seq]) * unit;
      const CacheSeq s = cache_seq(dm, cu_q, seq_lens, seq);
      for (int x = 0; x < 2; ++x) {
        const int n_tok = min(s.n - t0 - x * plan.tokens, plan.tokens);
        if (n_tok > 0) mine += (max(min(s.len - s.n_all + t0 + x * plan.tokens + n_tok, s.keys), 0) + kStep - 1) / kStep;
      }
      steps[tid] = mine;
    }
    __syncthreads();
    if (tid < units) {
      int ahead = 0;
      for (int v = 0; v < units; ++v) ahead += steps[v] > mine || (steps[v] == mine && v < tid);
      if (ahead == rank) { sm.seq = seq; sm.token0 = t0; }
    }
    fence_proxy_async_smem();                                  // (tiles will be copied over the table)
  } else if (warp == 0) {
    const int u = plan.units - 1 - rank;
    int seen = 0, seq = -1, t0 = 0;
    bool bad = false;
    const bool all = u == 0 && h == 0 && part == 0;      // (this CTA looks at every sequence, for the status word)
    for (int i0 = 0; i0 < dm.n_seq && (seq < 0 || all); i0 += 32) {
      const int i = i0 + lane;
      int n = 0;
      if (i < dm.n_seq) {
        const CacheSeq s = cache_seq(dm, cu_q, seq_lens, i);
        n = dm.n_tokens ? plan.by_unit(s.n + plan.tokens * 2 - 1) : 0;
        bad = bad || s.bad;
      }
      int upto = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      const unsigned in = __ballot_sync(0xffffffffu, u < seen + upto);
      if (in && seq < 0) {
        const int l = __ffs(in) - 1;
        seq = i0 + l;
        t0 = (u - seen - __shfl_sync(0xffffffffu, upto - n, l)) * plan.tokens * 2;
      }
      seen += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (bad) cache_status(status_word, HGA_STATUS_BAD_INDEX);
    if (lane == 0) { sm.seq = seq; sm.token0 = t0; }
  }
  auto init_barriers = [&]() {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&sm.full[i], kFill);
      mbar_init(&sm.empty[i], 2);
      mbar_init(&sm.raw_full[i], 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&sm.raw_empty[x], kFill);
      for (int b = 0; b < 2; ++b) {
        mbar_init(&sm.s_full[x][b], 1);
        mbar_init(&sm.p_full[x][b], 4);
      }
      mbar_init(&sm.drain[x], 1);
    }
    fence_barrier_init();
  };
  if (tid == 32) {
    sm.abort = sm.strange = sm.wide = 0;
    init_barriers();
  }
  __syncthreads();
  const int seq = sm.seq, token0 = sm.token0;
  if (seq < 0) {                               // fewer units than there could be
    pdl_launch_dependents();
    return;
  }
  const CacheSeq s = cache_seq(dm, cu_q, seq_lens, seq);
  const int pos0 = s.len - s.n_all;
  const int n_tok = min(s.n - token0, 2 * plan.tokens);        // of the unit
  const int first_lim = min(pos0 + token0, s.keys - 1), last_lim = min(pos0 + token0 + n_tok - 1, s.keys - 1);
  const int k0 = part * plan.sp.keys, k1 = split ? min(k0 + plan.sp.keys, last_lim + 1) : last_lim + 1;
  if (part > 0 && k0 >= k1) {
    pdl_launch_dependents();
    return;
  }
  // steps of each M-tile (the first one's rows see fewer keys)
  auto steps_of = [&](int x) {
    const int n = min(n_tok - x * plan.tokens, plan.tokens);
    if (n <= 0) return 0;
    const int end = min(k1, min(pos0 + token0 + x * plan.tokens + n - 1, s.keys - 1) + 1);
    return max(end - k0 + kStep - 1, 0) / kStep;
  };
  const int n0 = steps_of(0), n1 = steps_of(1), n_tiles = (max(n0, n1) + 1) / 2;

  // Q, rows that are none as zeros
  constexpr int C = D / 8;
  constexpr bool kScaled = FMT != kCacheBf16;
  // fp16: scales are 2^(code - 127 + kLift), in range from 2^-14 to 2^kTop
  constexpr int kLift = FMT == kCacheMx8 ? 4 : 2, kTop = FMT == kCacheMx8 ? 7 : 13;
  auto load_q = [&](bool f16) {
    if (warp == 10 || warp == 11) return;      // (they copy)
    constexpr int kLoaders = kThreads - 64, kAll = 2 * kTile * C, kAtOnce = (kAll + kLoaders - 1) / kLoaders;      // all of a thread's
    static_assert(kAtOnce <= 10, "registers");
    const int first = warp < 10 ? tid : tid - 64;
#pragma unroll 1
    for (int base = first; base < kAll; base += kLoaders * kAtOnce) {
      uint4 v[kAtOnce];
#pragma unroll
      for (int b = 0; b < kAtOnce; ++b) {
        const int i = base + b * kLoaders, row = i / C, c = i % C, x = row / kTile, r = row % kTile;
        const int t = dm.by_G(r), tok = x * plan.tokens + t;
        v[b] = make_uint4(0, 0, 0, 0);
        if (i < kAll && t < plan.tokens && tok < n_tok)
          v[b] = *reinterpret_cast<const uint4*>(Q + (s.q0 + token0 + tok) * dm.qs[0] + (h * dm.G + r - t * dm.G) * dm.qs[1] + c * 8);
      }
#pragma unroll
      for (int b = 0; b < kAtOnce; ++b) {
        const int i = base + b * kLoaders, row = i / C, c = i % C, x = row / kTile, r = row % kTile;
        if (i >= kAll) break;                  // (a whole warp)
        if (kScaled && f16) {
          // the row's largest to 2^14 .. 2^15, by a power of two that fp32 holds (and its inverse)
          uint32_t* w = &v[b].x;
          uint32_t big = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) big = max(big, max(w[k] & 0x7fffu, (w[k] >> 16) & 0x7fffu));
#pragma unroll
          for (int k = 1; k < C; k <<= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, k));
          const int up = max(min(127 + 14 - (int)(big >> 7), 100), -113);
          const float f = __uint_as_float((uint32_t)(127 + up) << 23);
          if (c == 0) sm.q_up[row] = (int8_t)up;
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = pack_f16(__uint_as_float(w[k] << 16) * f, __uint_as_float(w[k] & 0xffff0000u) * f);
        }
        *reinterpret_cast<uint4*>(sm.q[x] + piece<D>(r, c)) = v[b];
      }
    }
    fence_proxy_async_smem();
  };
  // first tile with keys hidden from the unit's first row
  const int first_dirty = max(first_lim + 1 - k0, 0) / kTile;
  // bf16: the cleaning warps have nothing to do until that tile's turn, which may be longer than a bounded wait lasts (some 10^7 keys).  The warp
  // that copies V meets them at a barrier then, or where it gives up.
  const bool cleaners_sleep = FMT == kCacheBf16 && first_dirty > 0 && first_dirty < n_tiles;
  constexpr int kMeet = (kFill + 1) * 32;
  auto barrier_arrive = [&]() { __syncwarp(); asm volatile("bar.arrive 1, %0;" ::"n"(kMeet) : "memory"); };
  auto barrier_sync = [&]() { __syncwarp(); asm volatile("bar.sync 1, %0;" ::"n"(kMeet) : "memory"); };
  // Copies of tile j: of K by warp 10, of V by warp 11.  False: a wait ran out.
  bool bad_page = false;
  auto copy_tile = [&](int j) {
    const bool is_v = warp == 11;
    const CUtensorMap* map = is_v ? &map_v : &map_k;
    const int boxes = kTile / plan.box;
    // lane's box `at`: its page (a page behind the last one arrives as zeros) and row there
    auto place = [&](int at, int& r) {
      const int key = k0 + j * kTile + at * plan.box;
      r = 0;
      if (key >= k1) return dm.n_pages;
      const int e = dm.by_page(key), page = table[seq * dm.table_stride + e];
      if (page < 0 || page >= dm.n_pages) { bad_page = true; return dm.n_pages; }
      r = key - e * dm.page;
      return page;
    };
    if (!kScaled) {
      const int at_ring = 2 * j + is_v, use = at_ring / NS, slot = at_ring - use * NS;
      if (!all_wait(&sm.empty[slot], (use & 1) ^ 1, abort)) return false;
      uint64_t* bar = is_v && j >= first_dirty ? &sm.raw_full[slot] : &sm.full[slot];
      if (lane == 0) mbar_arrive_expect_tx(bar, Sm::kTileBytes);
      else if (lane < 4 && bar == &sm.full[slot]) mbar_arrive(bar);
      __syncwarp();
      if (lane < boxes * (D / 64)) {
        const int box = lane % boxes, panel = lane / boxes;
        int r;
        const int page = place(box, r);
        tma_load_5d(sm.ring[slot] + panel * (kTile * 128) + box * plan.box * 128, map, bar, 0, r, panel, h, page);
      }
    } else {
      uint8_t* dst = sm.raw[is_v];
      uint64_t* bar = &sm.raw_full[FMT == kCacheMx8 && is_v && j >= first_dirty ? 2 : is_v];
      if (!all_wait(&sm.raw_empty[is_v], (j & 1) ^ 1, abort)) return false;
      if (lane == 0) mbar_arrive_expect_tx(bar, Sm::kRaw + Sm::kRawScales);
      __syncwarp();
      if (lane < boxes) {
        int r;
        const int page = place(lane, r);
        tma_load_5d(dst + lane * plan.box * cache_row_bytes(FMT, D), map, bar, 0, r, h, page, 0);
        const uint8_t* scales = (is_v ? V_scale : K_scale) + (((int64_t)page * dm.Hkv + h) * dm.page + r) * (D / 32);
        bulk_load(dst + Sm::kRaw + lane * plan.box * (D / 32), page < dm.n_pages ? scales : kNoScales, plan.box * (D / 32), bar);
      }
    }
    __syncwarp();
    return true;
  };
  // e4m3: NaN codes in V tile j that only some rows of the unit see become zeros, by the warp that copied it.  (The converting warps, which
  // have no registers to spare, took 6 to 34 us longer for a pass of 560 with this among their work.)
  auto clean_tile = [&](int j) {
    const int from = max(first_lim + 1 - (k0 + j * kTile), 0), to = min(k1 - (k0 + j * kTile), kTile);
    constexpr int kPieces = cache_row_bytes(FMT, D) / 16;
    if (!all_wait(&sm.raw_full[2], (j - first_dirty) & 1, abort)) return false;
#pragma unroll 4
    for (int i = from * kPieces + lane; i < to * kPieces; i += 32) {
      uint4* const at16 = reinterpret_cast<uint4*>(sm.raw[1]) + i;
      uint4 y = *at16;
      if (e4m3_nan(y.x) | e4m3_nan(y.y) | e4m3_nan(y.z) | e4m3_nan(y.w)) {
        uint32_t* e = &y.x;
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] &= ~((e4m3_nan(e[k]) >> 7) * 255u);
        *at16 = y;
        sm.strange = 1;
      }
    }
    mbar_arrive_warp(&sm.raw_full[1]);
    return true;
  };
  if (warp == 8) {
    tmem_alloc(&sm.tmem_base, kTmemCols);
    tmem_relinquish();
    __syncwarp();
  }
  // (the first tiles are on their way while Q is fetched)
  if ((warp == 10 || warp == 11) && n_tiles > 0) copy_tile(0);
  load_q(kScaled);
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (tid == 0) pdl_launch_dependents();
  const uint32_t tmem = sm.tmem_base;
  // Behind the last tile: every role is done, sm.abort, sm.strange and sm.wide are final.  True: once more, in bf16.
  bool f16 = kScaled;
  auto again = [&]() {
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (!kScaled || !f16 || !sm.wide || *abort) return false;
    f16 = false;
    if (warp == 8 || warp == 9) {
      // (the last commits may not have arrived yet)
      mma_commit_w(elect_one(), &sm.drain[warp - 8]);
      mbar_wait(&sm.drain[warp - 8], 0);
    }
    __syncwarp();
    __syncthreads();
    load_q(false);
    if (tid == 0) {
      sm.strange = 0;
      for (uint64_t* b = sm.full; b < sm.drain + 2; ++b) mbar_inval(b);
      init_barriers();
    }
    __syncthreads();
    return true;
  };

  if (warp < 8) {
    // ------------------------------------------------------------------ softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int x = warp >> 2, r = tid & 127;
    const int t = dm.by_G(r), tok = x * plan.tokens + t;
    const bool real = t < plan.tokens && tok < n_tok;
    const int lim = real ? min(pos0 + token0 + tok, s.keys - 1) : 0x7fffffff;
    const int head = h * dm.G + r - t * dm.G, row = s.q0 + token0 + tok;
    const int n = x ? n1 : n0;
    const int tile_lim = min(pos0 + token0 + x * plan.tokens, s.keys - 1);       // of the M-tile's first row
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lanes + x * kTile, o_addr = tmem + lanes + 2 * kTile + x * D;
    float m = kNoRef, l = 0.f;
    bool ok;
    do {
      const float to_log2 = dm.scale * 1.44269504088896340736f * (kScaled && f16 ? __uint_as_float((uint32_t)(127 - sm.q_up[x * kTile + r] - kLift) << 23) : 1.f);
      const uint64_t to_log2_2 = pack_f32x2(to_log2, to_log2);
      m = kNoRef;
      l = 0.f;
      ok = true;
      auto steps = [&](auto as_f16) {
        constexpr bool kF16 = decltype(as_f16)::value;
        // One weight in eight by the FMA pipe: chunk of 2048 495 -> 475 us, one in four 485, one in two 507.  Not where a quantised head_dim 128 leaves
        // too few issue slots (569 -> 580).
        constexpr bool kByFma = !kScaled || D == 64;
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
          ok = all_wait(&sm.s_full[x][j & 1], (j >> 1) & 1, abort);
          if (!ok) break;
          tc_fence_after_sync();
          const uint32_t buf = s_addr + (j & 1) * kStep;
          uint32_t v[2][32];
#pragma unroll
          for (int i = 0; i < 2; ++i) tmem_ld32(buf + 32 * i, v[i]);
          tmem_wait_ld();
          const int base = k0 + j * kStep;
          if (base + kStep - 1 > tile_lim) {
            const int seen = lim - base;           // columns up to it are visible
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (32 * i + e > seen) v[i][e] = 0xff800000u;
          }
          // The weights are computed with the reference at hand, while the row's largest logit is looked for; where that is too large (in the
          // first step, and seldom after it) they are computed again.
          float sum;
#pragma unroll 1
          for (;;) {
            const uint64_t neg_m = pack_f32x2(-m, -m);
            uint64_t sum2[2];
            float top[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t p[16];
              sum2[i] = pack_f32x2(0.f, 0.f);
              top[i] = __uint_as_float(v[i][0]);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float x0 = __uint_as_float(v[i][2 * e]), x1 = __uint_as_float(v[i][2 * e + 1]);
                top[i] = fmaxf(top[i], fmaxf(x0, x1));
                float a0, a1;
                unpack_f32x2(fma_f32x2(pack_f32x2(x0, x1), to_log2_2, neg_m), a0, a1);
                if (kByFma && (e & 7) == 5) {
                  exp2_by_fma(a0, a1);
                } else {
                  a0 = fast_exp2(a0);
                  a1 = fast_exp2(a1);
                }
                sum2[i] = add_f32x2(sum2[i], pack_f32x2(a0, a1));
                p[e] = kF16 ? pack_f16(a0, a1) : pack_bf16(a0, a1);
              }
              tmem_st16(buf + 16 * i, p);
            }
            float s0, s1;
            unpack_f32x2(add_f32x2(sum2[0], sum2[1]), s0, s1);
            sum = s0 + s1;
            const float mx = fmaxf(top[0], top[1]) * to_log2;
            if (!__any_sync(0xffffffffu, mx > m + kSlack)) break;
            const float now = fmaxf(m, mx - kLow), f = fast_exp2(m - now);
            m = now;
            l *= f;
            if (j > 0) {
              // O may be touched when P V of the step before is done
              ok = all_wait(&sm.s_full[x][(j + 1) & 1], ((j + 1) >> 1) & 1, abort);
              if (!ok) break;
              tc_fence_after_sync();
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                uint32_t o[16];
                tmem_ld16(o_addr + c, o);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tmem_st16(o_addr + c, o);
              }
            }
          }
          if (!ok) break;
          l += sum;
          tmem_wait_st();
          tc_fence_before_sync();
          mbar_arrive_warp(&sm.p_full[x][j & 1]);
        }
      };
      if (f16) steps(std::true_type{});
      else steps(std::false_type{});
      if (ok && n > 0) ok = all_wait(&sm.s_full[x][(n + 1) & 1], ((n + 1) >> 1) & 1, abort);      // P V of the last step
    } while (again());
    if (!*abort && n_tok > x * plan.tokens) {
      tc_fence_after_sync();
      const bool whole = !split || (plan.sp.unit ? last_lim + 1 : s.keys) <= plan.sp.keys;
      const int64_t all_rows = (int64_t)plan.sp.tokens * dm.Hq, out_row = (int64_t)row * dm.Hq + head;
      const int64_t part_row = part * all_rows + (int64_t)(plan.sp.unit ? row - s.q0 : row) * dm.Hq + head;
      const float down = f16 ? 1.f / (float)(1 << kLift) : 1.f;                   // (V's lift)
      const float inv = l > 0.f ? (whole ? 1.f / l : 1.f) * down : (l == 0.f ? 0.f : l);      // (NaN stays NaN)
      // Rows pass through shared memory (every copy and GEMM is done), so that a warp stores them piece after piece: a row per lane instead
      // took three times as long.
      constexpr int kPitch = D * 4 + 16;
      static_assert(8 * 32 * kPitch <= (int)(sizeof(sm.q) + sizeof(sm.ring)), "the rows of eight warps");
      uint8_t* const mine = sm.q[0] + warp * (32 * kPitch);
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        __syncwarp();
        if (n > 0) {
          tmem_ld32(o_addr + c, o);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0;
        }
        if (sm.strange && real) {
          const int end = min(lim + 1, k1);
          uint32_t nan = 0;                                  // of a quantised pool: a bit per column
          for (int key = max(first_lim + 1, k0); key < end; ++key) {
            const int e0 = dm.by_page(key), pr = key - e0 * dm.page, page = table[seq * dm.table_stride + e0];
            if (page < 0 || page >= dm.n_pages) continue;
            if (FMT == kCacheBf16) {
              const uint16_t* src = reinterpret_cast<const uint16_t*>(V) + page * dm.vs[0] + h * dm.vs[1] + pr * dm.vs[2] + c;
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (not_finite(src[e])) o[e] = __float_as_uint(__uint_as_float(o[e]) + __uint_as_float((uint32_t)src[e] << 16));
            } else {
              if (V_scale[(((int64_t)page * dm.Hkv + h) * dm.page + pr) * (D / 32) + (c >> 5)] == 255) nan = ~0u;
              if (FMT == kCacheMx8) {
                const uint8_t* src = V + page * dm.vs[0] + h * dm.vs[1] + pr * dm.vs[2] + c;
#pragma unroll 1
                for (int e = 0; e < 32; ++e) nan |= (src[e] & 127) == 127 ? 1u << e : 0u;
              }
            }
          }
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if ((nan >> e) & 1) o[e] = 0x7fc00000u;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * inv);
        if (whole) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = pack_bf16(__uint_as_float(o[8 * e + 2 * k]), __uint_as_float(o[8 * e + 2 * k + 1]));
            *reinterpret_cast<uint4*>(mine + lane * kPitch + c * 2 + e * 16) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint4*>(mine + lane * kPitch + c * 4 + e * 16) = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        }
      }
      __syncwarp();
      const int64_t to = !real ? -1 : whole ? (row * dm.os[0] + head * dm.os[1]) * 2 : part_row * (D * 4);      // bytes
      uint8_t* const out = whole ? reinterpret_cast<uint8_t*>(O) : reinterpret_cast<uint8_t*>(part_o);
      const int pieces = whole ? D / 8 : D / 4;           // of a row
#pragma unroll 4
      for (int i = lane; i < 32 * pieces; i += 32) {
        const int64_t at_row = __shfl_sync(0xffffffffu, to, i / pieces);
        if (at_row >= 0)
          *reinterpret_cast<uint4*>(out + at_row + i % pieces * 16) = *reinterpret_cast<const uint4*>(mine + i / pieces * kPitch + i % pieces * 16);
      }
      if (real && whole && LSE) LSE[out_row] = l > 0.f ? (m + log2f(l)) * 0.69314718055994530942f : (l == 0.f ? -INFINITY : l);
      if (real && !whole)
        *reinterpret_cast<float4*>(part_o + plan.sp.parts * all_rows * D + part_row * 4) = make_float4(m, l, l, 0.f);
    }
  } else if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssueRegs));
    do {
      if (warp < 10) {
        // ---------------------------------------------------------------- GEMMs (the whole warp stays together, one lane issues)
        const int x = warp - 8, n = x ? n1 : n0;
        const uint32_t lead = elect_one();
        constexpr uint32_t kBf16 = (1u << 7) | (1u << 10);      // formats of A and B: bf16, else fp16
        const uint32_t type = f16 ? kBf16 : 0;
        const uint32_t idesc_s = idesc_bf16_f32(128, kStep, 0, 0) ^ type, idesc_o = idesc_bf16_f32(128, D, 0, 1) ^ type;
        const uint64_t q_desc = smem_desc_sw128(smem_u32(sm.q[x]), 16, 1024);
        const uint64_t k_desc = smem_desc_sw128(smem_u32(sm.ring), 16, 1024), v_desc = smem_desc_sw128(smem_u32(sm.ring), kTile * 128, 1024);
        const uint32_t s_tmem = tmem + x * kTile, o_tmem = tmem + 2 * kTile + x * D;
        // a step is half a tile: 64 rows of 128 bytes per panel
        auto issue_s = [&](int half, int slot) {
          const uint64_t b = desc_advance(k_desc, slot * Sm::kTileBytes + half * (kStep * 128));
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            const uint32_t off = (i >> 2) * (kTile * 128) + (i & 3) * 32;
            mma_ss_w(lead, s_tmem + half * kStep, desc_advance(q_desc, off), desc_advance(b, off), idesc_s, i > 0);
          }
        };
        auto issue_pv = [&](int half, int slot, bool add) {
          const uint64_t b = desc_advance(v_desc, slot * Sm::kTileBytes + half * (kStep * 128));
#pragma unroll
          for (int i = 0; i < kStep / 16; ++i) mma_ts_w(lead, o_tmem, s_tmem + half * kStep + 8 * i, desc_advance(b, i * 2048), idesc_o, add || i > 0);
        };
        // Position in the ring of K(j) is 2j, of V(j) 2j + 1.  Both warps release every slot, whether its keys concern their M-tile or not,
        // and always by a commit.
        int slot = 0;
        uint32_t phase = 0;
        auto next = [&]() { if (++slot == NS) { slot = 0; phase ^= 1; } };
        bool ok = true;
        if (n_tiles > 0) {
          ok = all_wait(&sm.full[0], 0, abort);
          if (ok) {
            tc_fence_after_sync();
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
              if (half < n) issue_s(half, 0);
              mma_commit_w(lead, &sm.s_full[x][half]);
            }
            mma_commit_w(lead, &sm.empty[0]);
            next();
          }
        }
#pragma unroll 1
        for (int j = 0; ok && j < n_tiles; ++j) {
          const int v_slot = slot;
          const bool more = j + 1 < n_tiles;
          ok = all_wait(&sm.full[v_slot], phase, abort);
          next();
          const int k_slot = slot;
          if (ok && more) ok = all_wait(&sm.full[k_slot], phase, abort);
#pragma unroll 1
          for (int half = 0; ok && half < 2; ++half) {
            const int step = 2 * j + half;
            if (step >= n) break;
            ok = all_wait(&sm.p_full[x][half], j & 1, abort);
            if (!ok) break;
            tc_fence_after_sync();
            issue_pv(half, v_slot, step > 0);
            if (step + 2 < n) issue_s(half, k_slot);
            mma_commit_w(lead, &sm.s_full[x][half]);
          }
          if (!ok) break;
          mma_commit_w(lead, &sm.empty[v_slot]);
          if (more) {
            mma_commit_w(lead, &sm.empty[k_slot]);
            next();
          }
        }
      } else {
        // ---------------------------------------------------------------- copies (tile 0 went ahead)
        bool told = warp != 11 || !cleaners_sleep;
        for (int j = 0; j < n_tiles; ++j) {
          if (!told && j == first_dirty) { barrier_arrive(); told = true; }
          if ((j > 0 || f16 != kScaled) && !copy_tile(j)) break;
          if (FMT == kCacheMx8 && warp == 11 && j >= first_dirty && !clean_tile(j)) break;
        }
        if (!told) barrier_arrive();
        if (bad_page) cache_status(status_word, HGA_STATUS_BAD_INDEX);
        if (*abort && lane == 0) {
          // giving up: give the copies still in flight time to land before shared memory is released
          for (int it = 0; it < 64; ++it) __nanosleep(1000);
        }
      }
    } while (again());
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRestRegs));
    const int w = warp - 12;
    do {
      bool strange = false;
      if (FMT == kCacheBf16) {
        // ---------------------------------------------------------------- V tiles with hidden keys: a thread per key
        const int r = tid & 127;
        uint32_t parity = 0;                     // of each slot's raw_full
        if (cleaners_sleep) barrier_sync();
#pragma unroll 1
        for (int j = first_dirty; j < n_tiles; ++j) {
          const int slot = (2 * j + 1) % NS;
          if (!all_wait(&sm.raw_full[slot], (parity >> slot) & 1, abort)) break;
          parity ^= 1u << slot;
          const int key = k0 + j * kTile + r;
          if (key > first_lim) {
#pragma unroll 4
            for (int c = 0; c < C; ++c) {
              uint4* at16 = reinterpret_cast<uint4*>(sm.ring[slot] + piece<D>(r, c));
              if (key >= k1) {
                *at16 = make_uint4(0, 0, 0, 0);
                continue;
              }
              uint4 y = *at16;
              uint32_t* e = &y.x;
              bool odd = false;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                if (not_finite(e[i])) { e[i] &= 0xffff0000u; odd = true; }
                if (not_finite(e[i] >> 16)) { e[i] &= 0xffffu; odd = true; }
              }
              if (odd) { *at16 = y; strange = true; }
            }
          }
          fence_proxy_async_smem();
          mbar_arrive_warp(&sm.full[slot]);
        }
      } else {
        // ---------------------------------------------------------------- quantised tiles: converted from one buffer into another
        constexpr int LPR = cache_row_bytes(FMT, D) / 16;        // lanes of a row
        constexpr int RPI = 32 / LPR, kRows = kFill * RPI;       // rows of a warp's access, of all warps' (a multiple of 8)
        constexpr int kPairs = FMT == kCacheMx8 ? 2 : 4;         // 16-byte pieces of bf16 or fp16 that a lane's 16 bytes become
        const int in_row = lane % LPR, r0 = w * RPI + lane / LPR;
        bool wide = false;
        auto convert = [&](auto as_f16) {
          constexpr bool kF16 = decltype(as_f16)::value;
#pragma unroll 1
          for (int i_ring = 0; i_ring < 2 * n_tiles; ++i_ring) {
            const int use = i_ring / NS, slot = i_ring - use * NS, j = i_ring >> 1;
            const bool is_v = i_ring & 1;
            if (!all_wait(&sm.raw_full[i_ring & 1], (i_ring >> 1) & 1, abort) || !all_wait(&sm.empty[slot], (use & 1) ^ 1, abort)) break;
            const uint8_t* src = sm.raw[i_ring & 1] + r0 * cache_row_bytes(FMT, D) + in_row * 16;
            const uint8_t* scales = sm.raw[i_ring & 1] + Sm::kRaw + r0 * (D / 32) + (FMT == kCacheMx8 ? in_row >> 1 : in_row);
            uint8_t* dst = sm.ring[slot];
            const int end = k1 - (k0 + j * kTile) - r0, hidden = is_v ? first_lim - (k0 + j * kTile) - r0 : kTile;      // rows from `end` on are none
#pragma unroll
            for (int i = 0; i < kTile / kRows; ++i) {
              uint4 y = *reinterpret_cast<const uint4*>(src + i * kRows * cache_row_bytes(FMT, D));
              uint32_t sc = scales[i * kRows * (D / 32)];
              if (i * kRows >= end) {
                y = make_uint4(0, 0, 0, 0);
                sc = 127;
              }
              const uint32_t q[4] = {y.x, y.y, y.z, y.w};
              uint32_t o[4 * kPairs], mul;
              if (kF16) {
                const uint32_t e = sc - (127 - kLift - 15);
                mul = e * 0x04000400u;
                if (e - 1 >= kTop + 15) {          // out of range: zeros (2^-127 counts as zero), NaN, or a number that is too large or small
                  if (sc == 255 && i * kRows > hidden) { sc = 0; strange = true; }
                  mul = sc == 255 ? 0x7e007e00u : 0u;
                  wide = wide || (sc != 0 && sc != 255);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  if (FMT == kCacheMx8) e4m3x4_to_f16(q[k], o[k * kPairs], o[k * kPairs + 1]);
                  else e2m1x8_to_f16(q[k], o[k * kPairs], o[k * kPairs + 1], o[k * kPairs + 2 % kPairs], o[k * kPairs + 3 % kPairs]);
#pragma unroll
                  for (int z = 0; z < kPairs; ++z) o[k * kPairs + z] = mul_f16x2(o[k * kPairs + z], mul);
                }
              } else {
                if (sc == 255 && i * kRows > hidden) { sc = 0; strange = true; }
                mul = pair(scale_bits(sc));
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  if (FMT == kCacheMx8) {
                    o[k * kPairs] = mul_bf16x2(mul_bf16x2(e4m3_to_bf16_scaled(__byte_perm(q[k], 0, 0x1404)), kTwo120), mul);
                    o[k * kPairs + 1] = mul_bf16x2(mul_bf16x2(e4m3_to_bf16_scaled(__byte_perm(q[k], 0, 0x3424)), kTwo120), mul);
                    const uint32_t nan = e4m3_nan(q[k]);
                    o[k * kPairs] |= nan_halves(nan, false);
                    o[k * kPairs + 1] |= nan_halves(nan, true);
                  } else {
                    e2m1x4_to_bf16(q[k] & 0xffffu, o[k * kPairs], o[k * kPairs + 1]);
                    e2m1x4_to_bf16(q[k] >> 16, o[k * kPairs + 2 % kPairs], o[k * kPairs + 3 % kPairs]);
#pragma unroll
                    for (int z = 0; z < kPairs; ++z) o[k * kPairs + z] = mul_bf16x2(o[k * kPairs + z], mul);
                  }
                }
              }
              // (Storing the pieces so that no two lanes meet a bank takes selections that cost more than the conflicts: 581 against 567 us.)
#pragma unroll
              for (int k = 0; k < kPairs; ++k)
                *reinterpret_cast<uint4*>(dst + piece<D>(r0, kPairs * in_row + k) + i * kRows * 128) = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
            }
            fence_proxy_async_smem();
            mbar_arrive_warp(&sm.full[slot]);
            mbar_arrive_warp(&sm.raw_empty[i_ring & 1]);
          }
        };
        if (f16) convert(std::true_type{});
        else convert(std::false_type{});
        if (wide) sm.wide = 1;
      }
      if (strange) sm.strange = 1;
    } while (again());
  }

  // common exit
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && sm.abort && status_word) atomicOr(status_word, HGA_STATUS_WAIT_TIMEOUT);
  if ((warp == 8 || warp == 9) && sm.abort) {
    // given up: GEMMs already issued may still be writing tensor memory; wait (bounded) until the tensor pipe has run dry
    mma_commit_w(elect_one(), &sm.drain[warp - 8]);
    mbar_wait(&sm.drain[warp - 8], 0);
    __syncwarp();
  }
  __syncthreads();
  if (warp == 8) {
    tmem_dealloc(sm.tmem_base, kTmemCols);
  }
}

Plan plan_of(const CacheDims& dm) {
  Plan p;
  p.tokens = kTile / dm.G;
  p.by_unit = Div(2 * p.tokens);
  p.box = 8;
  while (p.box < kTile && dm.page % (2 * p.box) == 0) p.box *= 2;
  // sum over the sequences of ceil(n / unit) <= tokens / unit + sequences; no sequence has more than max_new
  const int64_t unit = 2 * p.tokens;
  p.units = (int)std::min<int64_t>(dm.n_tokens / unit + std::min(dm.n_seq, dm.n_tokens), dm.n_seq * ((dm.max_new + unit - 1) / unit));
  // What n units take, whole or in k parts, in steps of 64 keys: rounds of the device, a CTA's set-up and end (16 steps' time), the join
  const int n = (int)std::min<int64_t>((int64_t)p.units * dm.Hkv, 0x7fffffff), sms = 148;
  const double steps = dm.max_keys / 64.;
  auto cost = [&](int64_t n, int k) { return (double)((n * k + sms - 1) / sms) * (steps / k + 16) + (k > 1 ? 25 + 2 * k : 0); };
  struct Cut { int parts; double first, cost; };      // first: steps of the first part, and of all but the last
  auto best_cut = [&](int64_t n) {
    Cut best{1, steps, cost(n, 1)};
    for (int k = 2; k <= 64 && dm.max_keys / k >= 512; ++k)
      if (cost(n, k) < best.cost) best = Cut{k, steps / k, cost(n, k)};
    // Or two parts, the first of which takes an SM each, and the rest the second ones, `r` one after another, in the same time (16384 keys, 88
    // units: 217 us in three even parts, 201 so)
    if (n > sms / 2 && n < sms) {
      const int64_t r = (n + sms - n - 1) / (sms - n);
      const double first = (r * (steps + 16) - 16) / (r + 1), c = first + 16 + 25 + 4;
      if (first < steps - 8 && c < best.cost) best = Cut{2, first, c};
    }
    return best;
  };
  p.sp.cluster = false;
  p.sp.tokens = dm.n_tokens;
  p.sp.unit = p.sp.units = p.sp.full = 0;
  Cut cut{1, steps, 0};
  if (n < sms) {
    // few units: their keys are shared out, so that the device is full, the more the less even their lengths may be
    if (dm.n_seq == 1 || n == 0) {
      cut = best_cut(n);                                 // (n = 0: without tokens)
    } else {
      cut.parts = std::min((2 * sms + n - 1) / n, std::max(dm.max_keys / 512, 1));
      cut.first = steps / cut.parts;
    }
  } else if (dm.n_seq == 1 && n % sms) {
    // the last round's, where that takes 7 % off.  16384 keys, whole / so: 176 units 470 / 324 us, 224 units 468 / 439, 240 units 471 / 445.  (256
    // units, of which it should take 5 % off: 471 / 472.  The device is then busy to the end, at a lower clock.)
    const int full = n / sms * sms;
    const Cut tail = best_cut(n - full);
    if (tail.parts > 1 && cost(n - full, 1) - tail.cost >= 0.07 * cost(n, 1)) {
      cut = tail;
      p.sp.unit = (int)unit;
      p.sp.units = p.units;
      p.sp.full = full;
      p.sp.tokens = (int)std::min<int64_t>((int64_t)(p.units - full / dm.Hkv) * unit, dm.n_tokens);
    }
  }
  p.sp.keys = cut.parts == 1 ? (dm.max_keys + kTile - 1) / kTile * kTile : (int)std::ceil(cut.first * kStep / kTile) * kTile;
  p.sp.parts = std::max((dm.max_keys + p.sp.keys - 1) / p.sp.keys, 1);
  if (p.sp.parts == 1) p.sp.unit = p.sp.units = p.sp.full = 0;
  p.ranked = dm.n_seq > 1 && dm.n_seq <= kMaxRanked && p.units <= kMaxRanked && p.sp.parts == 1;
  return p;
}

template <int FMT, int D>
int launch_of(const CacheDims& dm, const Plan& plan, const void* Q, const int32_t* cu_q, const int32_t* seq_lens, const int32_t* table,
              const void* K, const void* V, const void* K_scale, const void* V_scale, void* O, float* LSE, void* workspace,
              int32_t* status_word, cudaStream_t st) {
  const int64_t ctas = plan.sp.full + ((int64_t)plan.units * dm.Hkv - plan.sp.full) * plan.sp.parts;
  if (ctas > 0x7fffffff) return HGA_ERR_SHAPE;
  CUtensorMap mk = {}, mv = {};
  int bad;
  if (FMT == kCacheBf16) {
    const uint32_t box[5] = {64, (uint32_t)plan.box, 1, 1, 1};
    const uint64_t dims[5] = {64, (uint64_t)dm.page, (uint64_t)(D / 64), (uint64_t)dm.Hkv, (uint64_t)dm.n_pages};
    const uint64_t sk[4] = {(uint64_t)dm.ks[2] * 2, 128, (uint64_t)dm.ks[1] * 2, (uint64_t)dm.ks[0] * 2};
    const uint64_t sv[4] = {(uint64_t)dm.vs[2] * 2, 128, (uint64_t)dm.vs[1] * 2, (uint64_t)dm.vs[0] * 2};
    bad = encode_tensor_map_bf16(&mk, K, 5, dims, sk, box, true, false) | encode_tensor_map_bf16(&mv, V, 5, dims, sv, box, true, false);
  } else {
    constexpr uint32_t kRow = cache_row_bytes(FMT, D);
    const uint32_t box[5] = {kRow, (uint32_t)plan.box, 1, 1, 1};
    const uint64_t dims[5] = {kRow, (uint64_t)dm.page, (uint64_t)dm.Hkv, (uint64_t)dm.n_pages, 1};
    const uint64_t sk[4] = {(uint64_t)dm.ks[2], (uint64_t)dm.ks[1], (uint64_t)dm.ks[0], 16};
    const uint64_t sv[4] = {(uint64_t)dm.vs[2], (uint64_t)dm.vs[1], (uint64_t)dm.vs[0], 16};
    bad = encode_tensor_map_u8(&mk, K, 5, dims, sk, box) | encode_tensor_map_u8(&mv, V, 5, dims, sv, box);
  }
  if (bad) return HGA_ERR_UNSUPPORTED;
  auto* kernel = k_cache_attn_sm100<FMT, D>;
  const size_t smem = sizeof(Smem<FMT, D>) + 1024;
  static_assert(sizeof(Smem<FMT, D>) + 1024 <= 232448, "shared memory of a CTA");
  const int rc = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem, true);
  if (rc) return rc;
  // the registers that the warps pass on to one another are those of the launch
  static std::atomic<int> regs{0};
  if (regs == 0) {
    cudaFuncAttributes a;
    const cudaError_t e = cudaFuncGetAttributes(&a, reinterpret_cast<const void*>(kernel));
    if (e != cudaSuccess) return record_cuda(e);
    regs = a.numRegs;
  }
  if (regs < (2 * kSoftmaxRegs + kIssueRegs + kRestRegs) / 4) return HGA_ERR_UNSUPPORTED;
  PdlLaunch cfg(dim3((unsigned)ctas), kThreads, smem, st, 0);
  const cudaError_t e = cudaLaunchKernelEx(&cfg.c, kernel, mk, mv, dm, plan, (const uint16_t*)Q, cu_q, seq_lens, table, (const uint8_t*)K,
                                           (const uint8_t*)V, (const uint8_t*)K_scale, (const uint8_t*)V_scale, (uint16_t*)O, LSE,
                                           (float*)workspace, status_word);
  count_launch(HGA_KERNELS_CACHE_TENSOR);
  return record_cuda(e);
}

}  // namespace

CacheSplit cache_tensor_split(const CacheDims& dm) { return plan_of(dm).sp; }

int launch_cache_attn_sm100(const CacheDims& dm, const void* Q, const int32_t* cu_q, const int32_t* seq_lens, const int32_t* table,
                            const void* K, const void* V, const void* K_scale, const void* V_scale, void* O, float* LSE, void* workspace,
                            int32_t* status_word, cudaStream_t st) {
  const Plan plan = plan_of(dm);
#define HGA_TENSOR(F) (dm.d == 128 ? launch_of<F, 128> : launch_of<F, 64>)
  auto* f = dm.format == kCacheBf16 ? HGA_TENSOR(kCacheBf16) : dm.format == kCacheMx8 ? HGA_TENSOR(kCacheMx8) : HGA_TENSOR(kCacheMx4);
#undef HGA_TENSOR
  const int rc = f(dm, plan, Q, cu_q, seq_lens, table, K, V, K_scale, V_scale, O, LSE, workspace, status_word, st);
  if (rc || plan.sp.parts == 1) return rc;
  return launch_cache_join(dm, plan.sp, cu_q, seq_lens, workspace, O, LSE, st);
}

}  // namespace hga
