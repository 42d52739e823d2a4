// hga_cache_attn for few query rows: generation steps, drafted tokens.
//
// A tile is up to 16 query rows of one (sequence, key/value head) -- new tokens x query heads of the group -- and a CTA takes a run
// of keys for it.  Its four warps take 16 or 32 keys at a time, in turn, straight from global memory into the registers of warp-level
// matrix instructions: nothing is shared between warps until the end, where their sums meet in shared memory.  What bounds it is the
// keys' and values' bytes; tcgen05's 128-row tiles would be padding here.
//
// How the operands come about without a transposition: the order in which a product sums over its inner axis is free, and so is the
// order of the columns of its result.  S = Q K^T: lane (g, c) = (lane / 4, lane % 4) of the instruction needs four numbers of key g
// per 16 elements of the head dimension; it takes them from 16-byte pieces of the row of its own, and Q's registers are laid out for
// the same order.  O^T = V^T P^T: P's registers are those of S as they are; a lane needs columns g of V for keys 2c, 2c+1, 2c+8, 2c+9
// in pairs of keys, so it loads its share of the columns of these four rows and pairs them up by byte permutations.
//
// Softmax: every warp has one reference per row, raised (and its sums rescaled) only when a logit exceeds it by 2^8, so that most
// steps have no exchange between lanes.  LSE is of the exact probabilities; O is divided by the sum of the rounded ones, a
// product with a column of ones.
#include <algorithm>
#include <cmath>

#include "hga_cache.cuh"
#include "hga_sm100.cuh"

namespace hga {

using namespace sm100;

namespace {

constexpr int kWarps = 4;
constexpr float kNoRef = -1e30f;      // reference of a row without a key: 2^(-inf - it) = 0
constexpr float kSlack = 8.f;         // log2 of how far a weight may exceed its reference's

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int W> __device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* p) {
  if (W == 4) {
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(p));
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  } else if (W == 2) {
    const uint2 x = __ldg(reinterpret_cast<const uint2*>(p));
    w[0] = x.x; w[1] = x.y;
  } else {
    w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
  }
}

// Where eight consecutive keys lie (page_size is a multiple of 8): byte offsets of the first one's rows, and its row of scales;
// k < 0: no page of the pool
struct Octet {
  int64_t k, v, s;
};

// A lane's share of a row of K (a quarter) and of V (an eighth): 16-byte pieces, the lanes' pieces next to one another
template <int FMT, int D>
struct Share {
  static constexpr int kRow = cache_row_bytes(FMT, D);
  static constexpr int KW = kRow / 16, VW = kRow / 32;          // 32-bit words
  static constexpr int KP = KW < 4 ? KW : 4, VP = VW < 4 ? VW : 4;      // words of a piece
  // element of the head dimension that lane c's local element e of K is, e = 0 .. D/4 - 1
  __device__ static __forceinline__ int k_element(int c, int e) {
    constexpr int per = D / 4 / (KW / KP);
    return (e / per) * 4 * per + c * per + e % per;
  }
  __device__ static __forceinline__ int v_element(int g, int e) {
    constexpr int per = D / 8 / (VW / VP);
    return (e / per) * 8 * per + g * per + e % per;
  }
};

// the value of one element of the cache (for the few that are looked at one by one)
template <int FMT>
__device__ float one_value(const uint8_t* row, const uint8_t* scale, int e) {
  if (FMT == kCacheBf16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[e] << 16);
  return scale[e >> 5] == 255 ? __uint_as_float(0x7fc00000u) : 0.f;      // (finite ones are not asked for)
}

template <int FMT, int D, int NT>
__global__ void __launch_bounds__(kWarps * 32, NT == 1 ? 4 : 3)
k_cache_rows(const CacheDims dm, const CacheSplit sp, int n_mt, const uint16_t* __restrict__ Q, const int32_t* __restrict__ cu_q,
             const int32_t* __restrict__ seq_lens, const int32_t* __restrict__ table, const uint8_t* __restrict__ K,
             const uint8_t* __restrict__ V, const uint8_t* __restrict__ K_scale, const uint8_t* __restrict__ V_scale,
             uint16_t* __restrict__ O, float* __restrict__ LSE, float* __restrict__ part_o, int32_t* status_word) {
  typedef Share<FMT, D> Sh;
  constexpr int kRowsTile = 8 * NT;
  constexpr int KS = FMT == kCacheBf16 ? 16 : 32, SUB = KS / 16;       // keys a warp takes at once
  constexpr int kUnit = FMT == kCacheBf16 ? 2 : 1;
  constexpr int kPitch = D + 4;
  typedef typename ScaleWord<D>::type SW;
  extern __shared__ __align__(16) uint8_t smem[];
  Octet* oct = reinterpret_cast<Octet*>(smem);                                     // [sp.keys / 8]
  float* sm_o = reinterpret_cast<float*>(smem + (size_t)(sp.keys / 8) * sizeof(Octet));      // [kWarps][kRowsTile][kPitch]
  __shared__ float sm_m[kWarps][kRowsTile], sm_l[kWarps][kRowsTile], sm_r[kWarps][kRowsTile];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  int at = blockIdx.x;
  const int mt = at % n_mt;  at /= n_mt;
  const int part = at % sp.parts;  at /= sp.parts;
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
  if (part > 0 && k0 >= k1) return;
  const int nk = max(k1 - k0, 0);

  for (int o = threadIdx.x; o < (nk + 7) / 8; o += kWarps * 32) {
    const int pos = k0 + o * 8, e = dm.by_page(pos), r = pos - e * dm.page;
    const int page = table[seq * dm.table_stride + e];
    Octet x{-1, -1, 0};
    if (page >= 0 && page < dm.n_pages) {
      x.k = (page * dm.ks[0] + h * dm.ks[1] + r * dm.ks[2]) * kUnit;
      x.v = (page * dm.vs[0] + h * dm.vs[1] + r * dm.vs[2]) * kUnit;
      x.s = (((int64_t)page * dm.Hkv + h) * dm.page + r) * (D / 32);
    } else {
      cache_status(status_word, HGA_STATUS_BAD_INDEX);
    }
    oct[o] = x;
  }

  // Q in registers, in K's order; a row's last visible key
  uint32_t qa[D / 16][2 * NT];
  int lim[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = row0 + n * 8 + g;
    const bool real = row < rows;
    const int t = real ? dm.by_G(row) : 0, head = h * dm.G + (row - t * dm.G);
    lim[n] = real ? min(pos0 + t, s.keys - 1) : 0x7fffffff;
    const uint16_t* q = Q + (s.q0 + t) * dm.qs[0] + head * dm.qs[1];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      uint2 x = make_uint2(0, 0);
      if (real) x = *reinterpret_cast<const uint2*>(q + Sh::k_element(c, 4 * i));
      qa[i][2 * n] = x.x;
      qa[i][2 * n + 1] = x.y;
    }
  }
  __syncthreads();

  const int64_t k_lane = g * dm.ks[2] * kUnit + c * (Sh::KP * 4);
  uint32_t kw[2 * SUB][Sh::KW], vw[4 * SUB][Sh::VW];
  uint32_t ksc[2 * SUB], vsc[4 * SUB];

  auto load_k = [&](int step) {
#pragma unroll
    for (int u = 0; u < 2 * SUB; ++u) {
      const int key = step * KS + u * 8;
#pragma unroll
      for (int i = 0; i < Sh::KW; ++i) kw[u][i] = 0;
      ksc[u] = 0x7f7f7f7fu;
      if (key + g < nk) {
        const Octet x = oct[key >> 3];
        if (x.k >= 0) {
          const uint8_t* p = K + x.k + k_lane;
#pragma unroll
          for (int i = 0; i < Sh::KW / Sh::KP; ++i) load_words<Sh::KP>(&kw[u][i * Sh::KP], p + i * (16 * Sh::KP));
          if (FMT != kCacheBf16) ksc[u] = __ldg(reinterpret_cast<const SW*>(K_scale + x.s + g * (D / 32)));
        }
      }
    }
  };
  auto load_v = [&](int step) {
#pragma unroll
    for (int j = 0; j < 4 * SUB; ++j) {
      const int key = step * KS + (j >> 1) * 8, in = 2 * c + (j & 1);
#pragma unroll
      for (int i = 0; i < Sh::VW; ++i) vw[j][i] = 0;
      vsc[j] = 0x7f7f7f7fu;
      if (key + in < nk) {
        const Octet x = oct[key >> 3];
        if (x.k >= 0) {
          const uint8_t* p = V + x.v + in * dm.vs[2] * kUnit + g * (Sh::VP * 4);
#pragma unroll
          for (int i = 0; i < Sh::VW / Sh::VP; ++i) load_words<Sh::VP>(&vw[j][i * Sh::VP], p + i * (32 * Sh::VP));
          if (FMT != kCacheBf16) vsc[j] = __ldg(reinterpret_cast<const SW*>(V_scale + x.s + in * (D / 32)));
        }
      }
    }
  };

  float o[NT][D / 16][4], ones[NT][4], m[NT], l[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m[n] = kNoRef;
    l[n] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) ones[n][i] = 0.f;
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][t][i] = 0.f;
  }
  const float to_log2 = dm.scale * 1.44269504088896340736f;
  bool strange = false;                 // a value hidden from some row of the tile is no finite number
  const int n_steps = (nk + KS - 1) / KS;
  if (warp < n_steps) load_k(warp);

#pragma unroll 1
  for (int step = warp; step < n_steps; step += kWarps) {
    load_v(step);
    float x[2 * SUB][4];
#pragma unroll
    for (int u = 0; u < 2 * SUB; ++u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[u][i] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint32_t b0, b1;
        if (FMT == kCacheBf16) {
          b0 = kw[u][(2 * i) % Sh::KW];
          b1 = kw[u][(2 * i + 1) % Sh::KW];
        } else if (FMT == kCacheMx8) {
          // block of piece i / 4 (16 bytes): 2 (i / 4) + c / 2
          const uint32_t mul = pair(scale_bits((ksc[u] >> (8 * (2 * (i / 4) + (c >> 1)))) & 255u));
          b0 = mul_bf16x2(mul_bf16x2(e4m3_to_bf16_scaled(__byte_perm(kw[u][i % Sh::KW], 0, 0x1404)), kTwo120), mul);
          b1 = mul_bf16x2(mul_bf16x2(e4m3_to_bf16_scaled(__byte_perm(kw[u][i % Sh::KW], 0, 0x3424)), kTwo120), mul);
        } else {
          const uint32_t mul = pair(scale_bits((ksc[u] >> (8 * (D == 128 ? c : c >> 1))) & 255u));
          e2m1x4_to_bf16((i & 1) ? kw[u][(i / 2) % Sh::KW] >> 16 : kw[u][(i / 2) % Sh::KW] & 0xffffu, b0, b1);
          b0 = mul_bf16x2(b0, mul);
          b1 = mul_bf16x2(b1, mul);
        }
        mma_16816(x[u], qa[i][0], NT == 2 ? qa[i][2 % (2 * NT)] : 0u, qa[i][1], NT == 2 ? qa[i][3 % (2 * NT)] : 0u, b0, b1);
      }
    }
    if (step + kWarps < n_steps) load_k(step + kWarps);

    // logits in units of log2, hidden ones -inf
#pragma unroll
    for (int u = 0; u < 2 * SUB; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[u][i] *= to_log2;
    const int base = k0 + step * KS;
    if (base + KS - 1 > first_lim) {
#pragma unroll
      for (int u = 0; u < 2 * SUB; ++u)
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i)
          if (base + u * 8 + 2 * c + (i & 1) > lim[i >> 1] || base + u * 8 + 2 * c + (i & 1) >= k1) x[u][i] = -INFINITY;
      // values hidden from the first row: a weight of zero does not silence an infinity, so such numbers are left out here and
      // given to the rows that see them at the end
#pragma unroll
      for (int j = 0; j < 4 * SUB; ++j) {
        if (base + (j >> 1) * 8 + 2 * c + (j & 1) <= first_lim) continue;
        if (FMT == kCacheBf16) {
#pragma unroll
          for (int i = 0; i < Sh::VW; ++i) {
            if ((vw[j][i] & 0x7f80u) == 0x7f80u) { vw[j][i] &= 0xffff0000u; strange = true; }
            if ((vw[j][i] & 0x7f800000u) == 0x7f800000u) { vw[j][i] &= 0xffffu; strange = true; }
          }
        } else {
#pragma unroll
          for (int i = 0; i < D / 32; ++i)
            if (((vsc[j] >> (8 * i)) & 255u) == 255u) { vsc[j] &= ~(255u << (8 * i)); strange = true; }
        }
      }
    }
    float top[NT];
    bool raise = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      top[n] = x[0][2 * n];
#pragma unroll
      for (int u = 0; u < 2 * SUB; ++u) top[n] = fmaxf(top[n], fmaxf(x[u][2 * n], x[u][2 * n + 1]));
      raise = raise || top[n] > m[n] + kSlack;
    }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float now = fmaxf(m[n], top[n]);
        now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, 1));
        now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, 2));
        const float f = fast_exp2(m[n] - now);
        m[n] = now;
        l[n] *= f;
        const float f0 = __shfl_sync(0xffffffffu, f, 8 * c), f1 = __shfl_sync(0xffffffffu, f, 8 * c + 4);      // of rows 2c, 2c + 1
#pragma unroll
        for (int i = 0; i < 4; ++i) ones[n][i] *= (i & 1) ? f1 : f0;
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][t][i] *= (i & 1) ? f1 : f0;
      }
    }
    uint32_t p[NT][2 * SUB];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int u = 0; u < 2 * SUB; ++u) {
        const float p0 = fast_exp2(x[u][2 * n] - m[n]), p1 = fast_exp2(x[u][2 * n + 1] - m[n]);
        l[n] += p0 + p1;
        p[n][u] = pack_bf16(p0, p1);
      }
#pragma unroll
    for (int b = 0; b < SUB; ++b) {
      uint32_t mul01 = 0, mul23 = 0;
      if (FMT != kCacheBf16) {
        const int sh = 8 * (D == 128 ? g >> 1 : g >> 2);
        mul01 = scale_bits((vsc[4 * b] >> sh) & 255u) | (scale_bits((vsc[4 * b + 1] >> sh) & 255u) << 16);
        mul23 = scale_bits((vsc[4 * b + 2] >> sh) & 255u) | (scale_bits((vsc[4 * b + 3] >> sh) & 255u) << 16);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
        mma_16816(ones[n], 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, p[n][2 * b], p[n][2 * b + 1]);
#pragma unroll
      for (int t = 0; t < D / 16; ++t) {      // local columns 2t, 2t + 1
        uint32_t a[4];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t* w0 = vw[4 * b + 2 * half];
          const uint32_t* w1 = vw[4 * b + 2 * half + 1];
          if (FMT == kCacheBf16) {
            a[2 * half] = __byte_perm(w0[t % Sh::VW], w1[t % Sh::VW], 0x5410);
            a[2 * half + 1] = __byte_perm(w0[t % Sh::VW], w1[t % Sh::VW], 0x7632);
          } else if (FMT == kCacheMx8) {
            const uint32_t mul = half ? mul23 : mul01;
            const uint32_t u0 = w0[(t / 2) % Sh::VW], u1 = w1[(t / 2) % Sh::VW];
            a[2 * half] = mul_bf16x2(mul_bf16x2(e4m3_to_bf16_scaled(__byte_perm(u0, u1, (t & 1) ? 0x6420 : 0x4400)), kTwo120), mul);
            a[2 * half + 1] = mul_bf16x2(mul_bf16x2(e4m3_to_bf16_scaled(__byte_perm(u0, u1, (t & 1) ? 0x7430 : 0x5410)), kTwo120), mul);
          } else {
            const uint32_t mul = half ? mul23 : mul01;
            const uint32_t u0 = w0[(t / 4) % Sh::VW], u1 = w1[(t / 4) % Sh::VW];
            const uint32_t even = (u0 & 0x0f0f0f0fu) | ((u1 << 4) & 0xf0f0f0f0u), odd = ((u0 >> 4) & 0x0f0f0f0fu) | (u1 & 0xf0f0f0f0u);
            uint32_t e0, e1, d0, d1;
            e2m1x4_to_bf16((t & 2) ? even >> 16 : even & 0xffffu, e0, e1);
            e2m1x4_to_bf16((t & 2) ? odd >> 16 : odd & 0xffffu, d0, d1);
            a[2 * half] = mul_bf16x2((t & 1) ? e1 : e0, mul);
            a[2 * half + 1] = mul_bf16x2((t & 1) ? d1 : d0, mul);
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_16816(o[n][t], a[0], a[1], a[2], a[3], p[n][2 * b], p[n][2 * b + 1]);
      }
    }
  }

  // the warps' sums meet
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    l[n] += __shfl_xor_sync(0xffffffffu, l[n], 1);
    l[n] += __shfl_xor_sync(0xffffffffu, l[n], 2);
    if (c == 0) { sm_m[warp][n * 8 + g] = m[n]; sm_l[warp][n * 8 + g] = l[n]; }
    if (g == 0) { sm_r[warp][n * 8 + 2 * c] = ones[n][0]; sm_r[warp][n * 8 + 2 * c + 1] = ones[n][1]; }
    float* dst = sm_o + (size_t)(warp * kRowsTile + n * 8 + 2 * c) * kPitch;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      const int col = Sh::v_element(g, 2 * t);
      *reinterpret_cast<float2*>(dst + col) = make_float2(o[n][t][0], o[n][t][2]);
      *reinterpret_cast<float2*>(dst + kPitch + col) = make_float2(o[n][t][1], o[n][t][3]);
    }
  }
  const bool any_strange = __syncthreads_or(strange);
  const bool whole = s.keys <= sp.keys;                  // the sequence is one part
  const int64_t all_rows = (int64_t)dm.n_tokens * dm.Hq;
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
      const float4 x = *reinterpret_cast<const float4*>(sm_o + (size_t)(w * kRowsTile + r) * kPitch + col);
      sum.x += f * x.x; sum.y += f * x.y; sum.z += f * x.z; sum.w += f * x.w;
      ls += f * sm_l[w][r];
      lr += f * sm_r[w][r];
    }
    const int t = dm.by_G(row), head = h * dm.G + (row - t * dm.G), tok = s.q0 + t;
    if (any_strange) {
      const int end = min(min(pos0 + t, s.keys - 1) + 1, k1);
      for (int key = max(first_lim + 1, k0); key < end; ++key) {
        const Octet x = oct[(key - k0) >> 3];
        if (x.k < 0) continue;
        const int in = (key - k0) & 7;
        const uint8_t* vr = V + x.v + in * dm.vs[2] * kUnit;
        const uint8_t* sr = V_scale + x.s + in * (D / 32);
        float* e = &sum.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y = one_value<FMT>(vr, sr, col + i);
          if (!isfinite(y)) e[i] += y;
        }
      }
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
}

// Joins the parts of every row: one warp per (token, query head)
template <int D>
__global__ void __launch_bounds__(256)
k_cache_join(const CacheDims dm, const CacheSplit sp, const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens,
             const float* __restrict__ part_o, uint16_t* __restrict__ O, float* __restrict__ LSE) {
  const int64_t all_rows = (int64_t)dm.n_tokens * dm.Hq;
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  pdl_wait();
  pdl_launch_dependents();
  if (row >= all_rows) return;
  const int tok = (int)(row / dm.Hq), head = (int)(row - (int64_t)tok * dm.Hq);
  int lo = 0, hi = dm.n_seq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu_q[mid] <= tok) lo = mid; else hi = mid;
  }
  const CacheSeq s = cache_seq(dm, cu_q, seq_lens, lo);
  if (tok < s.q0 || tok - s.q0 >= s.n || s.keys <= sp.keys) return;
  const int last = min(s.len - s.n_all + (tok - s.q0), s.keys - 1);
  const int parts = last < 0 ? 0 : last / sp.keys + 1;
  const float4* ml = reinterpret_cast<const float4*>(part_o + sp.parts * all_rows * D);
  float top = kNoRef;
  for (int i = lane; i < parts; i += 32) top = fmaxf(top, ml[i * all_rows + row].x);
#pragma unroll
  for (int i = 16; i; i >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
  constexpr int N = D / 32;
  float sum[N], ls = 0.f, lr = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.f;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) {
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
  const float inv = lr > 0.f ? 1.f / lr : (lr == 0.f ? 0.f : lr);
  uint32_t* dst = reinterpret_cast<uint32_t*>(O + tok * dm.os[0] + head * dm.os[1] + lane * N);
#pragma unroll
  for (int e = 0; e < N; e += 2) dst[e / 2] = pack_bf16(sum[e] * inv, sum[e + 1] * inv);
  if (LSE && lane == 0) LSE[row] = ls > 0.f ? (top + log2f(ls)) * 0.69314718055994530942f : (ls == 0.f ? -INFINITY : ls);
}

template <int FMT, int D, int NT>
int rows_of(const CacheDims& dm, const CacheSplit& sp, const void* Q, const int32_t* cu_q, const int32_t* seq_lens, const int32_t* table,
            const void* K, const void* V, const void* K_scale, const void* V_scale, void* O, float* LSE, void* workspace,
            int32_t* status_word, cudaStream_t st) {
  const int n_mt = (dm.max_new * dm.G + 8 * NT - 1) / (8 * NT);
  const int64_t ctas = (int64_t)dm.n_seq * dm.Hkv * sp.parts * n_mt;
  if (ctas > 0x7fffffff) return HGA_ERR_SHAPE;
  const size_t smem = (size_t)(sp.keys / 8) * sizeof(Octet) + (size_t)kWarps * 8 * NT * (D + 4) * sizeof(float);
  auto* kernel = k_cache_rows<FMT, D, NT>;
  const int rc = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem, true);
  if (rc) return rc;
  PdlLaunch cfg(dim3((unsigned)ctas), kWarps * 32, smem, st, 0);
  const cudaError_t e = cudaLaunchKernelEx(&cfg.c, kernel, dm, sp, n_mt, (const uint16_t*)Q, cu_q, seq_lens, table, (const uint8_t*)K,
                                           (const uint8_t*)V, (const uint8_t*)K_scale, (const uint8_t*)V_scale, (uint16_t*)O, LSE,
                                           (float*)workspace, status_word);
  count_launch(HGA_KERNELS_CACHE_ROWS);
  return record_cuda(e);
}

}  // namespace

// Keys per CTA: few enough that the device is full with the sequences as long as max_len says, many enough that a CTA's set-up does
// not show.  (Sequences are usually shorter; CTAs without keys cost next to nothing.)
CacheSplit cache_rows_split(const CacheDims& dm) {
  const int64_t tiles = (int64_t)dm.n_seq * dm.Hkv * ((dm.max_new * dm.G + 15) / 16);
  const int64_t want = (dm.max_keys * tiles + 148 * 6 - 1) / (148 * 6);
  CacheSplit sp;
  sp.keys = (int)std::min<int64_t>(std::max<int64_t>((want + 127) / 128 * 128, 256), 4096);
  sp.parts = std::max((dm.max_keys + sp.keys - 1) / sp.keys, 1);
  return sp;
}

int launch_cache_join(const CacheDims& dm, const CacheSplit& sp, const int32_t* cu_q, const int32_t* seq_lens, const void* workspace,
                      void* O, float* LSE, cudaStream_t st) {
  const int64_t rows = (int64_t)dm.n_tokens * dm.Hq;
  PdlLaunch cfg(dim3((unsigned)((rows + 7) / 8)), 256, 0, st, 0);
  const cudaError_t e = cudaLaunchKernelEx(&cfg.c, dm.d == 128 ? k_cache_join<128> : k_cache_join<64>, dm, sp, cu_q, seq_lens,
                                           (const float*)workspace, (uint16_t*)O, LSE);
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
  if (rc || sp.parts == 1) return rc;
  return launch_cache_join(dm, sp, cu_q, seq_lens, workspace, O, LSE, st);
}

}  // namespace hga
