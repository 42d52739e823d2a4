// hga_cache_write, hga_cache_read: new tokens into the paged cache, resident ones back as dense bf16.
//
// Both are streams: a thread has eight consecutive numbers of one row of K and the same ones of V, so that a warp's accesses are
// contiguous on the dense side (512 bytes) and, row by row, on the cache's.
#include "hga_cache.cuh"
#include "hga_sm100.cuh"

namespace hga {

using namespace sm100;

namespace {

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Scale code of a block whose largest magnitude has these bf16 bits (sign cleared): the smallest s >= 0 with amax <= top * 2^(s - 127), top
// = 1.75 * 2^8 or 1.5 * 2^2; 255 for infinities and NaN.  The exponent field of a subnormal counts as it is: s comes out as 0.
template <int FMT>
__device__ __forceinline__ int scale_code(uint32_t amax) {
  constexpr int kTopExp = FMT == kCacheMx8 ? 8 : 2, kTopMant = FMT == kCacheMx8 ? 96 : 64;
  const int e = (int)(amax >> 7), m = (int)(amax & 127);
  if (e == 255) return 255;
  return max(e - kTopExp + (m > kTopMant ? 1 : 0), 0);
}

// 2^(127 - s) for s in 0..254 (s = 0: 2^127; larger s may make it subnormal, down to 2^-127)
__device__ __forceinline__ float inverse_scale(int s) {
  return s <= 253 ? __uint_as_float((uint32_t)(254 - s) << 23) : __uint_as_float(1u << 22);
}

// two numbers -> two e4m3 bytes / two e2m1 nibbles (first in the low part), round to nearest even
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ uint32_t to_e2m1x2(float a, float b) {
  uint32_t r;
  asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// Eight numbers of a row into the cache.  The four threads of a block of 32 are neighbours in the warp and all here or all not.
template <int FMT>
__device__ __forceinline__ void put8(uint4 x, uint8_t* row, uint8_t* scale, int c, unsigned mask) {
  if (FMT == kCacheBf16) {
    *reinterpret_cast<uint4*>(row + c * 16) = x;
    return;
  }
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) amax = max(amax, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
  amax = max(amax, __shfl_xor_sync(mask, amax, 1));
  amax = max(amax, __shfl_xor_sync(mask, amax, 2));
  const int s = scale_code<FMT>(amax);
  // (past 2^127 times this the element would round to 2^128)
  const float most = FMT == kCacheMx8 ? (s == 247 ? 240.f : 448.f) : (s == 253 ? 3.f : 6.f);
  const float inv = s == 255 ? 0.f : inverse_scale(s);
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = fminf(fmaxf(bf16_lo(w[i]) * inv, -most), most);
    v[2 * i + 1] = fminf(fmaxf(bf16_hi(w[i]) * inv, -most), most);
  }
  if (FMT == kCacheMx8) {
    *reinterpret_cast<uint2*>(row + c * 8) = make_uint2(to_e4m3x2(v[0], v[1]) | (to_e4m3x2(v[2], v[3]) << 16),
                                                        to_e4m3x2(v[4], v[5]) | (to_e4m3x2(v[6], v[7]) << 16));
  } else {
    *reinterpret_cast<uint32_t*>(row + c * 4) = to_e2m1x2(v[0], v[1]) | (to_e2m1x2(v[2], v[3]) << 8) | (to_e2m1x2(v[4], v[5]) << 16) |
                                                (to_e2m1x2(v[6], v[7]) << 24);
  }
  if ((c & 3) == 0) scale[c >> 2] = (uint8_t)s;
}

template <int FMT, int D>
__global__ void __launch_bounds__(256)
k_cache_write(const CacheDims dm, const uint16_t* __restrict__ K_new, const uint16_t* __restrict__ V_new,
              const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens, const int32_t* __restrict__ table,
              uint8_t* __restrict__ K, uint8_t* __restrict__ V, uint8_t* __restrict__ K_scale, uint8_t* __restrict__ V_scale,
              int32_t* status_word, int n_rows) {
  constexpr int CH = D / 8;                     // threads of a row
  const int row = (int)(blockIdx.x * (256 / CH) + threadIdx.x / CH), c = threadIdx.x % CH;
  pdl_wait();
  pdl_launch_dependents();
  bool here = row < n_rows;                     // (CH divides the warp, so the threads of a row agree)
  const int t = here ? dm.by_Hkv(row) : 0, h = row - t * dm.Hkv;
  uint4 k = make_uint4(0, 0, 0, 0), v = k;
  if (here && K_new) k = *reinterpret_cast<const uint4*>(K_new + t * dm.kns[0] + h * dm.kns[1] + c * 8);
  if (here && V_new) v = *reinterpret_cast<const uint4*>(V_new + t * dm.vns[0] + h * dm.vns[1] + c * 8);
  // the sequence of token t: the last one that starts at or ahead of it
  int lo = 0, hi = dm.n_seq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu_q[mid] <= t) lo = mid; else hi = mid;
  }
  const CacheSeq s = cache_seq(dm, cu_q, seq_lens, lo);
  bool bad = s.bad;
  here = here && t >= s.q0 && t - s.q0 < s.n;
  const int pos = s.len - s.n_all + (t - s.q0);
  here = here && pos >= 0 && pos < dm.max_keys;
  int page = 0, r = 0;
  if (here) {
    const int e = dm.by_page(pos);
    r = pos - e * dm.page;
    page = table[lo * dm.table_stride + e];
    if (page < 0 || page >= dm.n_pages) { bad = true; here = false; }
  }
  if (bad && c == 0 && h == 0) cache_status(status_word, HGA_STATUS_BAD_INDEX);
  const unsigned mask = __ballot_sync(0xffffffffu, here);
  if (!here) return;
  const int64_t srow = (((int64_t)page * dm.Hkv + h) * dm.page + r) * (D / 32);
  constexpr int kUnit = FMT == kCacheBf16 ? 2 : 1;
  if (K_new) put8<FMT>(k, K + (page * dm.ks[0] + h * dm.ks[1] + r * dm.ks[2]) * kUnit, K_scale + srow, c, mask);
  if (V_new) put8<FMT>(v, V + (page * dm.vs[0] + h * dm.vs[1] + r * dm.vs[2]) * kUnit, V_scale + srow, c, mask);
}

// Eight numbers of a row out of the cache
template <int FMT> struct Raw8 { typedef uint4 type; };
template <> struct Raw8<kCacheMx8> { typedef uint2 type; };
template <> struct Raw8<kCacheMx4> { typedef uint32_t type; };

__device__ __forceinline__ uint4 take8(uint4 x, uint32_t) { return x; }
__device__ __forceinline__ uint4 take8(uint2 x, uint32_t scale) {
  const uint32_t m = pair(scale_bits(scale));
  auto two = [&](uint32_t w) { return mul_bf16x2(mul_bf16x2(e4m3_to_bf16_scaled(w), kTwo120), m); };
  return make_uint4(two(__byte_perm(x.x, 0, 0x1404)), two(__byte_perm(x.x, 0, 0x3424)), two(__byte_perm(x.y, 0, 0x1404)),
                    two(__byte_perm(x.y, 0, 0x3424)));
}
__device__ __forceinline__ uint4 take8(uint32_t x, uint32_t scale) {
  const uint32_t m = pair(scale_bits(scale));
  uint4 r;
  e2m1x4_to_bf16(x & 0xffffu, r.x, r.y);
  e2m1x4_to_bf16(x >> 16, r.z, r.w);
  return make_uint4(mul_bf16x2(r.x, m), mul_bf16x2(r.y, m), mul_bf16x2(r.z, m), mul_bf16x2(r.w, m));
}

constexpr int kReadRows = 4;      // rows a thread has in flight

template <int FMT, int D>
__global__ void __launch_bounds__(256)
k_cache_read(const CacheDims dm, int tok_begin, int n, const int32_t* __restrict__ seq_lens, const int32_t* __restrict__ table,
             const uint8_t* __restrict__ K, const uint8_t* __restrict__ V, const uint8_t* __restrict__ K_scale,
             const uint8_t* __restrict__ V_scale, uint16_t* __restrict__ K_out, uint16_t* __restrict__ V_out, int32_t* status_word,
             int blocks_per_head) {
  typedef typename Raw8<FMT>::type Raw;
  constexpr int CH = D / 8, kRows = 256 / CH;
  const int bh = blockIdx.x / blocks_per_head, blk = blockIdx.x - bh * blocks_per_head;
  const int i = dm.by_Hkv(bh), h = bh - i * dm.Hkv;
  const int c = threadIdx.x % CH, r0 = blk * (kRows * kReadRows) + threadIdx.x / CH;
  constexpr int kUnit = FMT == kCacheBf16 ? 2 : 1;
  pdl_wait();
  pdl_launch_dependents();
  const int len = seq_lens[i];
  bool bad = len < 0 || len > dm.max_keys;
  const int end = min(len, dm.max_keys) - tok_begin;      // rows of this sequence that are there
  Raw k[kReadRows], v[kReadRows];
  uint32_t ks[kReadRows], vs[kReadRows];
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    const int r = r0 + u * kRows;
    k[u] = Raw{};
    v[u] = Raw{};
    ks[u] = vs[u] = 127;
    if (r < n && r < end) {
      const int pos = tok_begin + r, e = dm.by_page(pos), pr = pos - e * dm.page;
      const int page = table[i * dm.table_stride + e];
      if (page < 0 || page >= dm.n_pages) { bad = true; continue; }
      const int64_t srow = (((int64_t)page * dm.Hkv + h) * dm.page + pr) * (D / 32) + (c >> 2);
      if (K_out) {
        k[u] = *reinterpret_cast<const Raw*>(K + (page * dm.ks[0] + h * dm.ks[1] + pr * dm.ks[2]) * kUnit + c * sizeof(Raw));
        if (FMT != kCacheBf16) ks[u] = K_scale[srow];
      }
      if (V_out) {
        v[u] = *reinterpret_cast<const Raw*>(V + (page * dm.vs[0] + h * dm.vs[1] + pr * dm.vs[2]) * kUnit + c * sizeof(Raw));
        if (FMT != kCacheBf16) vs[u] = V_scale[srow];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    const int r = r0 + u * kRows;
    if (r < n && r < end) {
      const int64_t at = i * dm.outs[0] + h * dm.outs[1] + r * dm.outs[2] + c * 8;
      if (K_out) *reinterpret_cast<uint4*>(K_out + at) = take8(k[u], ks[u]);
      if (V_out) *reinterpret_cast<uint4*>(V_out + at) = take8(v[u], vs[u]);
    }
  }
  if (bad && c == 0) cache_status(status_word, HGA_STATUS_BAD_INDEX);
}

template <int FMT, int D>
int write_of(const CacheDims& dm, const void* K_new, const void* V_new, const int32_t* cu_q, const int32_t* seq_lens,
             const int32_t* table, void* K, void* V, void* K_scale, void* V_scale, int32_t* status_word, cudaStream_t st) {
  const int n_rows = dm.n_tokens * dm.Hkv, per = 256 / (D / 8);
  PdlLaunch cfg(dim3((n_rows + per - 1) / per), 256, 0, st, 0);
  const cudaError_t e = cudaLaunchKernelEx(&cfg.c, k_cache_write<FMT, D>, dm, (const uint16_t*)K_new, (const uint16_t*)V_new, cu_q,
                                           seq_lens, table, (uint8_t*)K, (uint8_t*)V, (uint8_t*)K_scale, (uint8_t*)V_scale,
                                           status_word, n_rows);
  count_launch(HGA_KERNELS_CACHE);
  return record_cuda(e);
}

template <int FMT, int D>
int read_of(const CacheDims& dm, int tok_begin, int n, const int32_t* seq_lens, const int32_t* table, const void* K, const void* V,
            const void* K_scale, const void* V_scale, void* K_out, void* V_out, int32_t* status_word, cudaStream_t st) {
  constexpr int per = 256 / (D / 8) * kReadRows;
  const int blocks = (n + per - 1) / per;
  PdlLaunch cfg(dim3((unsigned)((int64_t)blocks * dm.n_seq * dm.Hkv)), 256, 0, st, 0);
  const cudaError_t e = cudaLaunchKernelEx(&cfg.c, k_cache_read<FMT, D>, dm, tok_begin, n, seq_lens, table, (const uint8_t*)K,
                                           (const uint8_t*)V, (const uint8_t*)K_scale, (const uint8_t*)V_scale, (uint16_t*)K_out,
                                           (uint16_t*)V_out, status_word, blocks);
  count_launch(HGA_KERNELS_CACHE);
  return record_cuda(e);
}

}  // namespace

int launch_cache_write(const CacheDims& dm, const void* K_new, const void* V_new, const int32_t* cu_q, const int32_t* seq_lens,
                       const int32_t* table, void* K, void* V, void* K_scale, void* V_scale, int32_t* status_word, cudaStream_t st) {
  auto* f = dm.format == kCacheBf16  ? (dm.d == 128 ? write_of<kCacheBf16, 128> : write_of<kCacheBf16, 64>)
            : dm.format == kCacheMx8 ? (dm.d == 128 ? write_of<kCacheMx8, 128> : write_of<kCacheMx8, 64>)
                                     : (dm.d == 128 ? write_of<kCacheMx4, 128> : write_of<kCacheMx4, 64>);
  return f(dm, K_new, V_new, cu_q, seq_lens, table, K, V, K_scale, V_scale, status_word, st);
}

int launch_cache_read(const CacheDims& dm, int tok_begin, int tok_end, const int32_t* seq_lens, const int32_t* table, const void* K,
                      const void* V, const void* K_scale, const void* V_scale, void* K_out, void* V_out, int32_t* status_word,
                      cudaStream_t st) {
  auto* f = dm.format == kCacheBf16  ? (dm.d == 128 ? read_of<kCacheBf16, 128> : read_of<kCacheBf16, 64>)
            : dm.format == kCacheMx8 ? (dm.d == 128 ? read_of<kCacheMx8, 128> : read_of<kCacheMx8, 64>)
                                     : (dm.d == 128 ? read_of<kCacheMx4, 128> : read_of<kCacheMx4, 64>);
  return f(dm, tok_begin, tok_end - tok_begin, seq_lens, table, K, V, K_scale, V_scale, K_out, V_out, status_word, st);
}

}  // namespace hga
