// hga_cache_attn for few query rows: generation steps, drafted tokens.
//
// A tile is up to 16 query rows of one (sequence, key/value head) -- new tokens x query heads of the group -- and a CTA takes a run
// of keys for it.  Its four warps take 16 or 32 keys at a time, in turn, each through a ring of its own in shared memory that
// cp.async fills ahead, and work on them with warp-level matrix instructions: nothing is shared between warps until the end, where
// their sums meet.  What bounds it is the keys' and values' bytes; tcgen05's 128-row tiles would be padding here.
//
// How the operands come about: S^T = K Q^T and O^T = V^T P^T, so that the few query rows are the short side (8 or 16) of both products;
// between them P^T is transposed in registers.  bf16: the registers of K and (transposed) of V are what ldmatrix delivers.
// Quantised: the order in which a product sums over its inner axis is free, and so is the order of the rows of its result, so a lane
// (g, c) = (lane / 4, lane % 4) takes eight numbers of every block of the keys g and g + 8, and Q's registers are laid out for the same
// order; of V it takes the columns g D/8 .. of the keys 2c, 2c+1, 2c+8, 2c+9 and pairs these up.
//
// Quantised pages are multiplied as fp16, into which the converter instructions go, and which holds e4m3 and e2m1 exactly.  K without
// its scales: they multiply the sums over a block (fp32) afterwards; Q is brought to fp16 by a power of two per row, exactly but for
// numbers 2^-29 of the row's largest.  V with its scales, times 2^kLift, where all of a step's lie in fp16's range (of blocks
// between 2^-12 and 2^9 in magnitude, e4m3; blocks of zeros need none); other steps go through bf16, exactly too, and slower.
//
// Softmax: every warp has one reference per row, raised (and its sums rescaled) only when a logit exceeds it by 2^14, so that most
// steps have no exchange between lanes.  It stays 2^6 below the row's largest when it is raised: fp16 then keeps weights down to 2^-31.
// LSE is of the exact probabilities; O is divided by the sum of the rounded ones, a product with a column of ones.
//
// Measured, 32 query heads on 8 of 128, one token: bf16, 65533 keys 48.8 us (5.5 TB/s, 84 % of a copy's rate); 32 sequences of 16K bf16 316 us
// (6.8 TB/s), e4m3 202 to 220 us from one machine to another (5.0 to 5.5 TB/s), e2m1 143 us (4.0 TB/s).  What has fewer bytes leaves every unit below
// its limit (e4m3: HBM 54 %, issue slots 44 %): latency, with three CTAs of four warps per SM, each with one step of copies ahead.
#include <algorithm>
#include <type_traits>

#include <cuda_fp16.h>

#include "hga_cache.cuh"
#include "hga_sm100.cuh"

namespace hga {

using namespace sm100;

namespace {

constexpr int kWarps = 4;
constexpr float kNoRef = -3e38f;      // reference of a row without a key: 2^(-inf - it) = 0, and any logit raises it
constexpr float kLow = 6.f, kSlack = 14.f;      // log2: how far the reference is set below the largest logit, and may be exceeded

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <bool kF16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (kF16) mma_f16(d, a0, a1, a2, a3, b0, b1);
  else mma_bf16(d, a0, a1, a2, a3, b0, b1);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void mma_f16_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {      // d = a b
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
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
// fp16 pairs that are bf16 numbers of few bits, as bf16 pairs
__device__ __forceinline__ uint32_t f16_to_bf16(uint32_t x) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x));
  return pack_bf16(f.x, f.y);
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {      // of a matrix of pairs, a row in four lanes
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {      // or zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <bool kTrans>
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  if (kTrans)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <int W>
__device__ __forceinline__ void lds(uint32_t* w, const uint8_t* p) {
  if (W == 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  } else if (W == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x; w[1] = x.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

constexpr int kMaxCluster = 8;
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// sixteen bytes at the address `here` (of this CTA's shared memory) in CTA `rank` of the cluster
__device__ __forceinline__ float4 peer_float4(uint32_t here, int rank) {
  float4 r;
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
               : "=f"(r.x), "=f"(r.y), "=f"(r.z), "=f"(r.w) : "r"(here), "r"(rank) : "memory");
  return r;
}

// Where eight consecutive keys lie (page_size is a multiple of 8): the first one's rows, and its row of scales; k null: no page of the pool
struct Octet {
  const uint8_t *k, *v;
  int64_t s;
};

// One warp's share of shared memory
template <int FMT, int D>
struct Ring {
  static constexpr int KS = FMT == kCacheBf16 ? 16 : 32;             // keys of a step
  static constexpr int kRow = cache_row_bytes(FMT, D), NP = kRow / 16;      // bytes and 16-byte pieces of a row
  static constexpr int kStages = 2;
  static constexpr int NB = D / 32;                                  // blocks of a row
  static constexpr int kScales = FMT == kCacheBf16 ? 0 : KS * NB;    // bytes
  static constexpr int kStage = 2 * KS * kRow + 2 * kScales;         // K, V, their scales
  static constexpr int kFactors = FMT == kCacheBf16 ? 0 : KS * NB * 6;      // K's scales as fp32 [key][block], V's as fp16 [block][key]
  static constexpr int kBytes = kStages * kStage + kFactors;
  // physical piece of piece p of row r, so that the accesses below meet no bank twice
  __device__ static __forceinline__ int k_piece(int r, int p) {
    if (FMT == kCacheBf16) return p ^ (r & 7);
    if (NP == 8) return p ^ ((r & 3) << 1);
    if (FMT == kCacheMx8) return p ^ (r & 2);
    return NP == 4 ? p ^ ((r >> 1) & 3) : p ^ ((r >> 2) & 1);
  }
  __device__ static __forceinline__ int v_piece(int r, int p) {
    if (FMT == kCacheBf16) return p ^ (r & 7);
    if (NP == 8) return p ^ (r & 6);
    return NP == 4 ? p ^ (r & 2) : p;
  }
};

// columns of O that rows g and g + 8 of product t are
template <int FMT, int D>
__device__ __forceinline__ int column(int g, int t, int half) {
  return FMT == kCacheBf16 ? 16 * t + 8 * half + g : g * (D / 8) + 2 * t + half;
}

// the value of one element, where it is not finite
template <int FMT>
__device__ float strange_value(const uint8_t* row, const uint8_t* scale, int e) {
  if (FMT == kCacheBf16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[e] << 16);
  return scale[e >> 5] == 255 || (FMT == kCacheMx8 && (row[e] & 127) == 127) ? __uint_as_float(0x7fc00000u) : 0.f;
}

template <int FMT, int D, int NT>
__global__ void __launch_bounds__(kWarps * 32, FMT == kCacheMx4 && NT == 1 ? 4 : 3)
k_cache_rows(const CacheDims dm, const CacheSplit sp, int n_mt, const uint16_t* Q, const int32_t* cu_q,
             const int32_t* seq_lens, const int32_t* table, const uint8_t* K,
             const uint8_t* V, const uint8_t* K_scale, const uint8_t* V_scale,
             uint16_t* O, float* LSE, float* part_o, int32_t* status_word) {
  typedef Ring<FMT, D> Rg;
  constexpr int kRowsTile = 8 * NT, KS = Rg::KS, SUB = KS / 16, NB = Rg::NB;
  constexpr int kUnit = FMT == kCacheBf16 ? 2 : 1;
  constexpr int kPitch = D + 4;
  constexpr bool kScaled = FMT != kCacheBf16;
  // V's scales are 2^(code - 127 + kLift) as fp16; in range: 2^-14 .. 2^kTop
  constexpr int kLift = FMT == kCacheMx8 ? 6 : FMT == kCacheMx4 ? 4 : 0, kTop = FMT == kCacheMx8 ? 7 : 13;
  static_assert(kRowsTile * kPitch * 4 <= Rg::kBytes, "a warp's sums take the place of its ring");
  extern __shared__ __align__(16) uint8_t smem[];
  Octet* oct = reinterpret_cast<Octet*>(smem);                                     // [sp.keys / 8]
  __shared__ float4 sm_part[kRowsTile];
  __shared__ float sm_m[kWarps][kRowsTile], sm_l[kWarps][kRowsTile], sm_r[kWarps][kRowsTile];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  uint8_t* const rings = smem + (size_t)(sp.keys / 8) * sizeof(Octet);
  uint8_t* const ring = rings + warp * Rg::kBytes;
  float* const k_factor = reinterpret_cast<float*>(ring + Rg::kStages * Rg::kStage);              // [KS][NB]
  uint16_t* const v_factor = reinterpret_cast<uint16_t*>(k_factor + KS * NB);                     // [NB][KS]
  // (parts that form a cluster follow one another; otherwise the tiles that read the same keys do)
  int at = blockIdx.x;
  const int inner = sp.cluster ? sp.parts : n_mt, outer = sp.cluster ? n_mt : sp.parts;
  const int at_inner = at % inner;  at /= inner;
  const int at_outer = at % outer;  at /= outer;
  const int mt = sp.cluster ? at_outer : at_inner, part = sp.cluster ? at_inner : at_outer;
  const int seq = dm.by_Hkv(at), h = at - seq * dm.Hkv;

  pdl_wait();
  pdl_launch_dependents();
  const CacheSeq s = cache_seq(dm, cu_q, seq_lens, seq);
  if (s.bad && threadIdx.x == 0 && h == 0 && part == 0 && mt == 0) cache_status(status_word, HGA_STATUS_BAD_INDEX);
  const int rows = s.n * dm.G, row0 = mt * kRowsTile;
  if (row0 >= rows) return;
  const int pos0 = s.len - s.n_all;                                    // position of the first new token
  const int last_row = min(rows, row0 + kRowsTile) - 1;
  const int first_lim = min(pos0 + dm.by_G(row0), s.keys - 1);         // last key that the tile's first row sees
  const int k0 = part * sp.keys;
  const int k1 = min(k0 + sp.keys, min(pos0 + dm.by_G(last_row), s.keys - 1) + 1);
  if (part > 0 && k0 >= k1 && !sp.cluster) return;
  const int nk = max(k1 - k0, 0);

  bool all_there = true;
  for (int o = threadIdx.x; o < (nk + 7) / 8; o += kWarps * 32) {
    const int pos = k0 + o * 8, e = dm.by_page(pos), r = pos - e * dm.page;
    const int page = table[seq * dm.table_stride + e];
    Octet x{nullptr, nullptr, 0};
    if (page >= 0 && page < dm.n_pages) {
      x.k = K + (page * dm.ks[0] + h * dm.ks[1] + r * dm.ks[2]) * kUnit;
      x.v = V + (page * dm.vs[0] + h * dm.vs[1] + r * dm.vs[2]) * kUnit;
      x.s = (((int64_t)page * dm.Hkv + h) * dm.page + r) * NB;
    } else {
      cache_status(status_word, HGA_STATUS_BAD_INDEX);
      all_there = false;
    }
    oct[o] = x;
  }

  // Q in registers, in K's order; a row's last visible key; what its logits are multiplied by
  uint32_t qa[D / 16][2 * NT];
  int lim[NT][2];                       // of rows 2c, 2c + 1
  float to_log2[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = row0 + n * 8 + 2 * c + i;
      lim[n][i] = row < rows ? min(pos0 + dm.by_G(row), s.keys - 1) : 0x7fffffff;
    }
    float per_row = dm.scale * 1.44269504088896340736f;      // of row g
    const int row = row0 + n * 8 + g;
    const bool real = row < rows;
    const int t = real ? dm.by_G(row) : 0, head = h * dm.G + (row - t * dm.G);
    const uint16_t* q = Q + (s.q0 + t) * dm.qs[0] + head * dm.qs[1];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      qa[i][2 * n] = qa[i][2 * n + 1] = 0;
      if (!real) continue;
      if (kScaled) {
        const uint2 x = *reinterpret_cast<const uint2*>(q + (i >> 1) * 32 + c * 8 + (i & 1) * 4);
        qa[i][2 * n] = x.x;
        qa[i][2 * n + 1] = x.y;
      } else {
        qa[i][2 * n] = *reinterpret_cast<const uint32_t*>(q + 16 * i + 2 * c);
        qa[i][2 * n + 1] = *reinterpret_cast<const uint32_t*>(q + 16 * i + 8 + 2 * c);
      }
    }
    if (kScaled) {
      uint32_t big = 0;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int k = 2 * n; k < 2 * n + 2; ++k) big = max(big, max(qa[i][k] & 0x7fffu, (qa[i][k] >> 16) & 0x7fffu));
      big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
      // the row's largest to 2^14 .. 2^15, by a power of two that fp32 holds (and its inverse)
      const int up = max(min(127 + 14 - (int)(big >> 7), 100), -113);
      const float f = __uint_as_float((uint32_t)(127 + up) << 23);
      per_row *= __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int k = 2 * n; k < 2 * n + 2; ++k)
          qa[i][k] = pack_f16(__uint_as_float(qa[i][k] << 16) * f, __uint_as_float(qa[i][k] & 0xffff0000u) * f);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) to_log2[n][i] = __shfl_sync(0xffffffffu, per_row, 8 * c + 4 * i);
  }
  all_there = __syncthreads_and(all_there);

  // Copies of one step: a lane's 16-byte pieces are those of number i * 32 + lane, row by row.  Keys past the end, and pages that are
  // none, become zeros; steps without any need no test.
  const uint32_t ring_addr = smem_u32(ring);
  constexpr int kIter = KS * Rg::NP / 32, RPI = 32 / Rg::NP;             // copies of a lane, of K and of V; rows of a warp's
  const int lr = lane / Rg::NP, lp = lane % Rg::NP;
  const int64_t k_row = dm.ks[2] * kUnit, v_row = dm.vs[2] * kUnit;
  const int64_t k_lane = (lr & 7) * k_row + lp * 16, v_lane = (lr & 7) * v_row + lp * 16;
  constexpr int kPieces = KS * NB / 16;                                  // pieces of K's scales (eight keys have NB / 2), and of V's
  auto fetch = [&](int step, int stage) {
    const uint32_t dst = ring_addr + stage * Rg::kStage;
    const Octet* first = oct + step * (KS / 8);
    const bool whole = all_there && (step + 1) * KS <= nk;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const int r = i * RPI + lr;
      const Octet* x = first + i * RPI / 8 + (RPI > 8 ? lr >> 3 : 0);
      const uint32_t k_dst = dst + r * Rg::kRow + Rg::k_piece(r, lp) * 16, v_dst = dst + (KS + r) * Rg::kRow + Rg::v_piece(r, lp) * 16;
      if (whole) {
        copy16(k_dst, x->k + k_lane + (i * RPI & 7) * k_row);
        copy16(v_dst, x->v + v_lane + (i * RPI & 7) * v_row);
      } else {
        const bool there = step * KS + r < nk && x->k;
        copy16(k_dst, there ? x->k + k_lane + (i * RPI & 7) * k_row : K, there);
        copy16(v_dst, there ? x->v + v_lane + (i * RPI & 7) * v_row : V, there);
      }
    }
    if (kScaled && lane < 2 * kPieces) {
      const int i = lane % kPieces, o8 = i / (NB / 2);
      const Octet* x = first + o8;
      const bool there = step * KS + o8 * 8 < nk && x->k;
      copy16(dst + 2 * KS * Rg::kRow + lane * 16, (lane < kPieces ? K_scale : V_scale) + (there ? x->s + i % (NB / 2) * 16 : 0), there);
    }
  };

  float o[NT][D / 16][4], ones[NT][4], m[NT][2], l[NT][2];      // columns 2c, 2c + 1
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m[n][0] = m[n][1] = kNoRef;
    l[n][0] = l[n][1] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) ones[n][i] = 0.f;
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][t][i] = 0.f;
  }
  bool strange = false;                 // a value hidden from some row of the tile is no finite number
  const int n_steps = (nk + KS - 1) / KS;
  int ahead = warp, stage = 0;          // next step to fetch; stage of the step at hand
#pragma unroll
  for (int i = 0; i < Rg::kStages - 1; ++i) {
    if (ahead < n_steps) fetch(ahead, i);
    copies_commit();
    ahead += kWarps;
  }

#pragma unroll 1
  for (int step = warp; step < n_steps; step += kWarps) {
    copies_wait<Rg::kStages - 2>();
    __syncwarp();
    // (every lane is done with the stage of the step before, which is filled next)
    if (ahead < n_steps) fetch(ahead, stage == 0 ? Rg::kStages - 1 : stage - 1);
    copies_commit();
    ahead += kWarps;
    uint8_t* const buf = ring + stage * Rg::kStage;
    const uint8_t* const vbuf = buf + KS * Rg::kRow;
    const uint32_t buf_addr = ring_addr + stage * Rg::kStage;
    if (++stage == Rg::kStages) stage = 0;
    const int base = k0 + step * KS;
    const bool masked = base + KS - 1 > first_lim;

    bool fits = true;                   // V's scales are in fp16's range
    if (kScaled) {
      // a lane prepares the scales of key `lane`
      const uint8_t* sc = buf + 2 * KS * Rg::kRow;
      uint32_t wk, wv;
      if (NB == 4) {
        wk = *reinterpret_cast<const uint32_t*>(sc + lane * 4);
        wv = *reinterpret_cast<const uint32_t*>(sc + KS * NB + lane * 4);
      } else {
        wk = *reinterpret_cast<const uint16_t*>(sc + lane * 2);
        wv = *reinterpret_cast<const uint16_t*>(sc + KS * NB + lane * 2);
      }
      float f[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        // (2^-127 becomes zero: such a block adds less than 2^-118 |q| to a logit)
        f[b] = __uint_as_float(((wk >> (8 * b)) & 255u) << 23);
        const uint32_t e = ((wv >> (8 * b)) & 255u) - (127 - kLift - 15);      // fp16's exponent field
        fits = fits && e - 1 < kTop + 15;
        v_factor[b * KS + lane] = (uint16_t)(e << 10);
      }
      // (a byte of 255: NaN)
      if (((~wk - 0x01010101u) & wk & (NB == 4 ? 0x80808080u : 0x8080u)) != 0) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
          if (((wk >> (8 * b)) & 255u) == 255) f[b] = __uint_as_float(0x7fc00000u);
      }
      if (NB == 4) *reinterpret_cast<float4*>(k_factor + lane * 4) = make_float4(f[0], f[1], f[2 % NB], f[3 % NB]);
      else *reinterpret_cast<float2*>(k_factor + lane * 2) = make_float2(f[0], f[1]);
      fits = __all_sync(0xffffffffu, fits);
      __syncwarp();
    }
    if (FMT != kCacheMx4 && masked && first_lim + 1 < k1) {
      // Values that only some of the rows see: a weight of zero does not silence an infinity or a NaN, so such numbers are left out here and
      // given to the rows that see them at the end.  (Scales of 255: below.  From k1 on there are zeros.)
      for (int i = lane; i < KS * Rg::NP; i += 32) {
        const int r = i / Rg::NP;
        if (base + r <= first_lim) continue;
        uint4* y = reinterpret_cast<uint4*>(buf + KS * Rg::kRow + i * 16);
        uint4 x = *y;
        uint32_t* w = &x.x;
        bool odd = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (FMT == kCacheMx8) {
            const uint32_t nan = e4m3_nan(w[k]);
            w[k] &= ~((nan >> 7) * 255u);
            odd = odd || nan;
          } else {
            if ((w[k] & 0x7f80u) == 0x7f80u) { w[k] &= 0xffff0000u; odd = true; }
            if ((w[k] & 0x7f800000u) == 0x7f800000u) { w[k] &= 0xffffu; odd = true; }
          }
        }
        if (odd) { *y = x; strange = true; }
      }
      __syncwarp();
    }

    // keys (b 16 + g) and (.. + 8), rows 2c and 2c + 1
    float x[SUB][NT][4];
#pragma unroll
    for (int b = 0; b < SUB; ++b) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[b][n][i] = 0.f;
      if (!kScaled) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {        // (keys 0-7, 16i ..), (keys 8-15, 16i ..), (keys 0-7, 16i + 8 ..), (keys 8-15, 16i + 8 ..)
          uint32_t k[4];
          const int r = b * 16 + (lane & 15);
          ldmatrix4<false>(k, buf_addr + r * Rg::kRow + Rg::k_piece(r, 2 * i + (lane >> 4)) * 16);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_bf16(x[b][n], k[0], k[1], k[2], k[3], qa[i][2 * n], qa[i][2 * n + 1]);
        }
      } else {
        float f[2][NB];                           // of keys g, g + 8
#pragma unroll
        for (int i = 0; i < 2; ++i)
          lds<NB>(reinterpret_cast<uint32_t*>(f[i]), reinterpret_cast<const uint8_t*>(k_factor + (b * 16 + 8 * i + g) * NB));
#pragma unroll
        for (int t = 0; t < NB; ++t) {
          uint32_t k[2][4];                       // [16 elements][..]
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int r = b * 16 + 8 * i + g;
            if (FMT == kCacheMx8) {
              uint32_t w[2];
              lds<2>(w, buf + r * Rg::kRow + Rg::k_piece(r, 2 * t + (c >> 1)) * 16 + (c & 1) * 8);
              e4m3x4_to_f16(w[0], k[0][i], k[0][2 + i]);
              e4m3x4_to_f16(w[1], k[1][i], k[1][2 + i]);
            } else {
              uint32_t w;
              lds<1>(&w, buf + r * Rg::kRow + Rg::k_piece(r, t) * 16 + c * 4);
              e2m1x8_to_f16(w, k[0][i], k[0][2 + i], k[1][i], k[1][2 + i]);
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float acc[4];
            mma_f16_zero(acc, k[0][0], k[0][1], k[0][2], k[0][3], qa[2 * t][2 * n], qa[2 * t][2 * n + 1]);
            mma_f16(acc, k[1][0], k[1][1], k[1][2], k[1][3], qa[2 * t + 1][2 * n], qa[2 * t + 1][2 * n + 1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[b][n][i] = fmaf(acc[i], f[i >> 1][t], x[b][n][i]);
          }
        }
      }
    }

    // hidden logits -inf
    if (masked) {
#pragma unroll
      for (int b = 0; b < SUB; ++b)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = base + b * 16 + 8 * (i >> 1) + g;
            if (key > lim[n][i & 1] || key >= k1) x[b][n][i] = -INFINITY;
          }
    }
    float top[NT][2];
    bool raise = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        top[n][i] = fmaxf(x[0][n][i], x[0][n][i + 2]);
#pragma unroll
        for (int b = 1; b < SUB; ++b) top[n][i] = fmaxf(top[n][i], fmaxf(x[b][n][i], x[b][n][i + 2]));
        top[n][i] *= to_log2[n][i];     // (in units of log2)
        raise = raise || top[n][i] > m[n][i] + kSlack;
      }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float f[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float now = top[n][i];
#pragma unroll
          for (int k = 4; k < 32; k <<= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, k));
          now = fmaxf(m[n][i], now - kLow);
          f[i] = fast_exp2(m[n][i] - now);
          m[n][i] = now;
          l[n][i] *= f[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) ones[n][i] *= f[i & 1];
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][t][i] *= f[i & 1];
      }
    }
#pragma unroll
    for (int b = 0; b < SUB; ++b)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[b][n][i] = fast_exp2(fmaf(x[b][n][i], to_log2[n][i & 1], -m[n][i & 1]));
          l[n][i & 1] += x[b][n][i];
        }

    if (!kScaled) {
      uint32_t p[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) p[n][u] = transpose8x8(pack_bf16(x[0][n][2 * u], x[0][n][2 * u + 1]));
#pragma unroll
      for (int n = 0; n < NT; ++n) mma_bf16(ones[n], 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, p[n][0], p[n][1]);
#pragma unroll
      for (int t = 0; t < D / 16; ++t) {
        // (keys 0-7, columns 16t ..), (same, 16t + 8 ..), (keys 8-15, 16t ..), (same, 16t + 8 ..), transposed
        uint32_t a[4];
        const int r = (lane & 7) + ((lane >> 4) << 3);
        ldmatrix4<true>(a, buf_addr + KS * Rg::kRow + r * Rg::kRow + Rg::v_piece(r, 2 * t + ((lane >> 3) & 1)) * 16);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_bf16(o[n][t], a[0], a[1], a[2], a[3], p[n][0], p[n][1]);
      }
    } else {
      constexpr int VW = Rg::kRow / 32;           // 32-bit words of a lane's share of a row of V
      const int block = g * NB / 8;
      auto weigh = [&](auto as_f16) {
        constexpr bool kF16 = decltype(as_f16)::value;
#pragma unroll
        for (int b = 0; b < SUB; ++b) {
          uint32_t w[4][VW], p[NT][2], mul[2];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int r = b * 16 + (j >> 1) * 8 + 2 * c + (j & 1), byte = g * 4 * VW;
            lds<VW>(w[j], vbuf + r * Rg::kRow + Rg::v_piece(r, byte >> 4) * 16 + (byte & 15));
          }
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int r = b * 16 + half * 8 + 2 * c;
            if (kF16) {
              mul[half] = *reinterpret_cast<const uint32_t*>(v_factor + block * KS + r);
            } else {
              // the scales as they are; the lift comes in by P
              const uint8_t* sc = buf + 2 * KS * Rg::kRow + KS * NB;
              uint32_t s0 = sc[r * NB + block], s1 = sc[(r + 1) * NB + block];
              // (NaN, hidden from some row: see above)
              if (s0 == 255 && base + r > first_lim) { s0 = 0; strange = true; }
              if (s1 == 255 && base + r + 1 > first_lim) { s1 = 0; strange = true; }
              mul[half] = scale_bits(s0) | (scale_bits(s1) << 16);
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
              p[n][u] = transpose8x8(kF16 ? pack_f16(x[b][n][2 * u], x[b][n][2 * u + 1]) : pack_bf16(x[b][n][2 * u], x[b][n][2 * u + 1]));
            constexpr uint32_t one = kF16 ? 0x3c003c00u : 0x3f803f80u;
            mma<kF16>(ones[n], one, one, one, one, p[n][0], p[n][1]);
            if (!kF16)
              for (int u = 0; u < 2; ++u) p[n][u] = mul_bf16x2(p[n][u], pack_bf16((float)(1 << kLift), (float)(1 << kLift)));
          }
#pragma unroll
          for (int t2 = 0; t2 < D / 32; ++t2) {      // local columns 4 t2 .. 4 t2 + 3
            uint32_t a[2][4];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t u0 = w[2 * half][t2 / (FMT == kCacheMx8 ? 1 : 2)], u1 = w[2 * half + 1][t2 / (FMT == kCacheMx8 ? 1 : 2)];
              uint32_t y[4];
              if (FMT == kCacheMx8) {
                e4m3x4_to_f16(__byte_perm(u0, u1, 0x5140), y[0], y[1]);
                e4m3x4_to_f16(__byte_perm(u0, u1, 0x7362), y[2], y[3]);
              } else {
                const uint32_t even = (u0 & 0x0f0f0f0fu) | ((u1 << 4) & 0xf0f0f0f0u), odd = ((u0 >> 4) & 0x0f0f0f0fu) | (u1 & 0xf0f0f0f0u);
                uint32_t e[4], d[4];               // (of a word each; the other half serves the next t2)
                e2m1x8_to_f16(even, e[0], e[1], e[2], e[3]);
                e2m1x8_to_f16(odd, d[0], d[1], d[2], d[3]);
                y[0] = e[2 * (t2 & 1)]; y[1] = d[2 * (t2 & 1)]; y[2] = e[2 * (t2 & 1) + 1]; y[3] = d[2 * (t2 & 1) + 1];
              }
#pragma unroll
              for (int k = 0; k < 4; ++k) a[k >> 1][2 * half + (k & 1)] = kF16 ? mul_f16x2(y[k], mul[half]) : mul_bf16x2(f16_to_bf16(y[k]), mul[half]);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int n = 0; n < NT; ++n) mma<kF16>(o[n][2 * t2 + k], a[k][0], a[k][1], a[k][2], a[k][3], p[n][0], p[n][1]);
          }
        }
      };
      if (!fits) {
        // What lies behind the last key, numbers that are zeros here, decides nothing; neither does 2^-127, the scale of a block of zeros and of
        // pages that are none, which becomes zero.  (Here, off the way of most steps: asked with the other scales it took 2 % longer.)
        bool others = true;
#pragma unroll 1
        for (int b = 0; b < NB; ++b) {
          const uint32_t code = base + lane < k1 ? buf[2 * KS * Rg::kRow + KS * NB + lane * NB + b] : 0u;
          if (code == 0) v_factor[b * KS + lane] = 0;
          else others = others && code - (127 - kLift - 15) - 1 < kTop + 15;
        }
        fits = __all_sync(0xffffffffu, others);
        __syncwarp();
      }
      if (fits) weigh(std::true_type{});
      else weigh(std::false_type{});
    }
  }
  copies_wait<0>();
  __syncwarp();

  // the warps' sums meet (each warp's in the place of its ring)
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int k = 4; k < 32; k <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], k);
      if (g == 0) {
        sm_m[warp][n * 8 + 2 * c + i] = m[n][i];
        sm_l[warp][n * 8 + 2 * c + i] = l[n][i];
        sm_r[warp][n * 8 + 2 * c + i] = ones[n][i];
      }
    }
    float* dst = reinterpret_cast<float*>(ring) + (n * 8 + 2 * c) * kPitch;
    constexpr float down = 1.f / (float)(1 << kLift);
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) dst[(i & 1) * kPitch + column<FMT, D>(g, t, i >> 1)] = o[n][t][i] * down;
  }
  const bool any_strange = __syncthreads_or(strange);
  const bool whole = s.keys <= sp.keys;                  // the sequence is one part
  const int64_t all_rows = (int64_t)sp.tokens * dm.Hq;
  constexpr int kCols = D / 4;                           // threads of a row
  for (int r = threadIdx.x / kCols; r < kRowsTile; r += kWarps * 32 / kCols) {
    const int row = row0 + r, col = (threadIdx.x % kCols) * 4;
    if (row >= rows) break;
    float top = sm_m[0][r];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) top = fmaxf(top, sm_m[w][r]);
    float4 sum = make_float4(0, 0, 0, 0);
    float ls = 0.f, lr = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = fast_exp2(sm_m[w][r] - top);
      const float4 x = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(rings + w * Rg::kBytes) + r * kPitch + col);
      sum.x += f * x.x; sum.y += f * x.y; sum.z += f * x.z; sum.w += f * x.w;
      ls += f * sm_l[w][r];
      lr += f * sm_r[w][r];
    }
    const int t = dm.by_G(row), head = h * dm.G + (row - t * dm.G), tok = s.q0 + t;
    if (any_strange) {
      const int end = min(min(pos0 + t, s.keys - 1) + 1, k1);
      for (int key = max(first_lim + 1, k0); key < end; ++key) {
        const Octet x = oct[(key - k0) >> 3];
        if (!x.k) continue;
        const int in = (key - k0) & 7;
        const uint8_t* vr = x.v + in * dm.vs[2] * kUnit;
        const uint8_t* sr = V_scale + x.s + in * (D / 32);
        float* e = &sum.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y = strange_value<FMT>(vr, sr, col + i);
          if (!isfinite(y)) e[i] += y;
        }
      }
    }
    if (sp.cluster) {
      // (in place: this thread alone reads here)
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(rings) + r * kPitch + col) = sum;
      if (col == 0) sm_part[r] = make_float4(top, ls, lr, 0.f);
      continue;
    }
    if (whole) {
      const float inv = lr > 0.f ? 1.f / lr : (lr == 0.f ? 0.f : lr);      // (NaN stays NaN)
      *reinterpret_cast<uint2*>(O + tok * dm.os[0] + head * dm.os[1] + col) =
          make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
      if (LSE && col == 0) LSE[(int64_t)tok * dm.Hq + head] = ls > 0.f ? (top + log2f(ls)) * 0.69314718055994530942f : (ls == 0.f ? -INFINITY : ls);
    } else {
      const int64_t at_row = part * all_rows + (int64_t)tok * dm.Hq + head;
      *reinterpret_cast<float4*>(part_o + at_row * D + col) = sum;
      if (col == 0) *reinterpret_cast<float4*>(part_o + sp.parts * all_rows * D + at_row * 4) = make_float4(top, ls, lr, 0.f);
    }
  }
  if (!sp.cluster) return;
  // the cluster's sums meet: each CTA finishes some of the rows
  cluster_sync();
  for (int r = part + sp.parts * (threadIdx.x / kCols); r < kRowsTile; r += sp.parts * (kWarps * 32 / kCols)) {
    const int row = row0 + r, col = (threadIdx.x % kCols) * 4;
    if (row >= rows) break;
    const uint32_t here = smem_u32(&sm_part[r]), sums = smem_u32(reinterpret_cast<float*>(rings) + r * kPitch + col);
    float4 ml[kMaxCluster];
    float top = kNoRef;
#pragma unroll
    for (int p = 0; p < kMaxCluster; ++p)
      if (p < sp.parts) {
        ml[p] = peer_float4(here, p);
        top = fmaxf(top, ml[p].x);
      }
    float4 sum = make_float4(0, 0, 0, 0);
    float ls = 0.f, lr = 0.f;
#pragma unroll
    for (int p = 0; p < kMaxCluster; ++p)
      if (p < sp.parts) {
        const float f = fast_exp2(ml[p].x - top);
        const float4 x = peer_float4(sums, p);
        sum.x += f * x.x; sum.y += f * x.y; sum.z += f * x.z; sum.w += f * x.w;
        ls += f * ml[p].y;
        lr += f * ml[p].z;
      }
    const int t = dm.by_G(row), head = h * dm.G + (row - t * dm.G), tok = s.q0 + t;
    const float inv = lr > 0.f ? 1.f / lr : (lr == 0.f ? 0.f : lr);
    *reinterpret_cast<uint2*>(O + tok * dm.os[0] + head * dm.os[1] + col) = make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
    if (LSE && col == 0) LSE[(int64_t)tok * dm.Hq + head] = ls > 0.f ? (top + log2f(ls)) * 0.69314718055994530942f : (ls == 0.f ? -INFINITY : ls);
  }
  cluster_sync();                       // nobody's shared memory goes while it is read
}

// Joins the parts of every (token, query head): W of a CTA's warps share the parts of a row out among them.  Eight where there are many parts
// of few rows (103 parts of 32 rows: one warp each took 35 us longer), one where there are few of many (4 parts of 28672 rows: eight took
// 130 us longer).
constexpr int kJoinWarps = 8;

template <int D, int W>
__global__ void __launch_bounds__(kJoinWarps * 32)
k_cache_join(const CacheDims dm, const CacheSplit sp, const int32_t* cu_q, const int32_t* seq_lens,
             const float* part_o, uint16_t* O, float* LSE) {
  constexpr int N = D / 32;
  __shared__ float sm_o[W][D], sm_l[W], sm_r[W], sm_m[W];
  const int64_t all_rows = (int64_t)sp.tokens * dm.Hq;      // of the partial results
  const int warp = (threadIdx.x >> 5) % W, lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * (kJoinWarps / W) + (threadIdx.x >> 5) / W;
  pdl_wait();
  pdl_launch_dependents();
  if (row >= all_rows) return;
  const int r_tok = (int)(row / dm.Hq), head = (int)(row - (int64_t)r_tok * dm.Hq);
  const CacheSeq s = cache_seq(dm, cu_q, seq_lens, sp.unit ? 0 : find_seq(cu_q, dm.n_seq, r_tok));
  const int tok = sp.unit ? s.q0 + r_tok : r_tok;
  if (tok < s.q0 || tok - s.q0 >= s.n) return;
  int keys = s.keys;                    // that what was written as one was decided by
  if (sp.unit) {
    const int u = r_tok / sp.unit;
    if ((sp.units - 1 - u) * dm.Hkv + dm.by_G(head) < sp.full) return;
    keys = min(s.len - s.n_all + min((u + 1) * sp.unit, s.n), s.keys);
  }
  if (keys <= sp.keys) return;
  const int last = min(s.len - s.n_all + (tok - s.q0), s.keys - 1);
  const int parts = last < 0 ? 0 : last / sp.keys + 1;
  const float4* ml = reinterpret_cast<const float4*>(part_o + sp.parts * all_rows * D);
  // each warp against the largest reference of its own parts
  float top = kNoRef;
  for (int i = warp + W * lane; i < parts; i += W * 32) top = fmaxf(top, ml[i * all_rows + row].x);
#pragma unroll
  for (int i = 16; i; i >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
  float sum[N], ls = 0.f, lr = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.f;
#pragma unroll 4
  for (int i = warp; i < parts; i += W) {
    const float4 x = ml[i * all_rows + row];
    const float f = fast_exp2(x.x - top);
    ls += f * x.y;
    lr += f * x.z;
    const float* src = part_o + (i * all_rows + row) * D + lane * N;
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float2 y = *reinterpret_cast<const float2*>(src + e);
      sum[e] += f * y.x;
      sum[e + 1] += f * y.y;
    }
  }
  uint16_t* const out = O + tok * dm.os[0] + head * dm.os[1];
  float* const lse = LSE ? LSE + (int64_t)tok * dm.Hq + head : nullptr;
  if (W == 1) {
    const float inv = lr > 0.f ? 1.f / lr : (lr == 0.f ? 0.f : lr);
#pragma unroll
    for (int e = 0; e < N; e += 2) *reinterpret_cast<uint32_t*>(out + lane * N + e) = pack_bf16(sum[e] * inv, sum[e + 1] * inv);
    if (lse && lane == 0) *lse = ls > 0.f ? (top + log2f(ls)) * 0.69314718055994530942f : (ls == 0.f ? -INFINITY : ls);
    return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e) sm_o[warp][lane * N + e] = sum[e];
  if (lane == 0) { sm_m[warp] = top; sm_l[warp] = ls; sm_r[warp] = lr; }
  __syncthreads();
  if (threadIdx.x >= D / 2) return;
  top = sm_m[0];
#pragma unroll
  for (int w = 1; w < W; ++w) top = fmaxf(top, sm_m[w]);
  float a = 0.f, b = 0.f;
  ls = lr = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float f = fast_exp2(sm_m[w] - top);
    a += f * sm_o[w][2 * threadIdx.x];
    b += f * sm_o[w][2 * threadIdx.x + 1];
    ls += f * sm_l[w];
    lr += f * sm_r[w];
  }
  const float inv = lr > 0.f ? 1.f / lr : (lr == 0.f ? 0.f : lr);
  *reinterpret_cast<uint32_t*>(out + 2 * threadIdx.x) = pack_bf16(a * inv, b * inv);
  if (lse && threadIdx.x == 0) *lse = ls > 0.f ? (top + log2f(ls)) * 0.69314718055994530942f : (ls == 0.f ? -INFINITY : ls);
}

template <int FMT, int D, int NT>
int rows_of(const CacheDims& dm, const CacheSplit& sp, const void* Q, const int32_t* cu_q, const int32_t* seq_lens, const int32_t* table,
            const void* K, const void* V, const void* K_scale, const void* V_scale, void* O, float* LSE, void* workspace,
            int32_t* status_word, cudaStream_t st) {
  const int n_mt = (dm.max_new * dm.G + 8 * NT - 1) / (8 * NT);
  const int64_t ctas = (int64_t)dm.n_seq * dm.Hkv * sp.parts * n_mt;
  if (ctas > 0x7fffffff) return HGA_ERR_SHAPE;
  const size_t smem = (size_t)(sp.keys / 8) * sizeof(Octet) + (size_t)kWarps * Ring<FMT, D>::kBytes;
  auto* kernel = k_cache_rows<FMT, D, NT>;
  const int rc = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem, true);
  if (rc) return rc;
  PdlLaunch cfg(dim3((unsigned)ctas), kWarps * 32, smem, st, 0);
  cudaLaunchAttribute attrs[2];
  if (sp.cluster) {
    attrs[0] = cfg.attr;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = sp.parts;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cfg.c.attrs = attrs;
    cfg.c.numAttrs = 2;
  }
  const cudaError_t e = cudaLaunchKernelEx(&cfg.c, kernel, dm, sp, n_mt, (const uint16_t*)Q, cu_q, seq_lens, table, (const uint8_t*)K,
                                           (const uint8_t*)V, (const uint8_t*)K_scale, (const uint8_t*)V_scale, (uint16_t*)O, LSE,
                                           (float*)workspace, status_word);
  count_launch(HGA_KERNELS_CACHE_ROWS);
  return record_cuda(e);
}

}  // namespace

// Keys per CTA: few enough that the device is full once with the sequences as long as max_len says, many enough that a CTA's set-up does
// not show, and no more than leave three CTAs' shared memory on an SM (e4m3, 32 sequences of 16K: 225 us with 2048, 201 with 1536).  (Sequences are usually shorter; CTAs without keys cost next to nothing.)
CacheSplit cache_rows_split(const CacheDims& dm) {
  const int64_t tiles = (int64_t)dm.n_seq * dm.Hkv * ((dm.max_new * dm.G + 15) / 16);
  const int64_t want = (dm.max_keys * tiles + 148 * 3 - 1) / (148 * 3);
  CacheSplit sp;
  sp.keys = (int)std::min<int64_t>(std::max<int64_t>((want + 127) / 128 * 128, 256), dm.format == kCacheMx8 ? 1536 : 2048);
  // Clusters for what is on the device at one time anyway: a CTA without keys keeps its place until its cluster is done.  There, latency
  // alone counts.
  const int64_t at_once = 148 * 2;
  if (dm.max_keys <= kMaxCluster * 128 && tiles * ((dm.max_keys + 127) / 128) <= at_once) sp.keys = 128;
  sp.parts = std::max((dm.max_keys + sp.keys - 1) / sp.keys, 1);
  sp.cluster = sp.parts > 1 && sp.parts <= kMaxCluster && tiles * sp.parts <= at_once;
  sp.tokens = dm.n_tokens;
  sp.unit = sp.units = sp.full = 0;
  return sp;
}

int launch_cache_join(const CacheDims& dm, const CacheSplit& sp, const int32_t* cu_q, const int32_t* seq_lens, const void* workspace,
                      void* O, float* LSE, cudaStream_t st) {
  const int64_t rows = (int64_t)sp.tokens * dm.Hq;
  const bool many = sp.parts > 16 || rows < 148 * 8;
  auto* kernel = many ? (dm.d == 128 ? k_cache_join<128, kJoinWarps> : k_cache_join<64, kJoinWarps>) : (dm.d == 128 ? k_cache_join<128, 1> : k_cache_join<64, 1>);
  PdlLaunch cfg(dim3((unsigned)(many ? rows : (rows + kJoinWarps - 1) / kJoinWarps)), kJoinWarps * 32, 0, st, 0);
  const cudaError_t e = cudaLaunchKernelEx(&cfg.c, kernel, dm, sp, cu_q, seq_lens, (const float*)workspace, (uint16_t*)O, LSE);
  count_launch(HGA_KERNELS_CACHE_ROWS);
  return record_cuda(e);
}

int launch_cache_attn_rows(const CacheDims& dm, const CacheSplit& sp, const void* Q, const int32_t* cu_q, const int32_t* seq_lens,
                           const int32_t* table, const void* K, const void* V, const void* K_scale, const void* V_scale, void* O,
                           float* LSE, void* workspace, int32_t* status_word, cudaStream_t st) {
  const bool one = dm.max_new * dm.G <= 8;
#define HGA_ROWS(F) (dm.d == 128 ? (one ? rows_of<F, 128, 1> : rows_of<F, 128, 2>) : (one ? rows_of<F, 64, 1> : rows_of<F, 64, 2>))
  auto* f = dm.format == kCacheBf16 ? HGA_ROWS(kCacheBf16) : dm.format == kCacheMx8 ? HGA_ROWS(kCacheMx8) : HGA_ROWS(kCacheMx4);
#undef HGA_ROWS
  const int rc = f(dm, sp, Q, cu_q, seq_lens, table, K, V, K_scale, V_scale, O, LSE, workspace, status_word, st);
  if (rc || sp.parts == 1 || sp.cluster) return rc;
  return launch_cache_join(dm, sp, cu_q, seq_lens, workspace, O, LSE, st);
}

}  // namespace hga
