// hga_cache_write, hga_cache_read: new tokens into the paged cache, resident ones back as dense bf16.
//
// Both are streams, bound by instructions as much as by bytes.  A thread has eight numbers of either half of a row of K and the same ones of
// V, and several rows: the lanes of a row access whole sectors on both sides, and where a row lies is worked out once for the four pieces.
//
// Measured, 8 heads of 128, calls one after another: 16384 tokens written in e4m3 in 20.0 to 20.8 us (102 MB, 4.9 to 5.1 TB/s; 72 % of the issue
// slots), in bf16 23.2 us (134 MB, 88 % of a copy's rate); 4 x 16384 read in e4m3 in 65.4 to 66.2 us (407 MB, 6.2 TB/s, 94 %), in e2m1 56.0
// (92 %), in bf16 83.9 (97 %).  One token each of 32 sequences: 9.1 to 9.8 us, of which the kernel has little more than the launch.
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
  // magnitudes compare as 16-bit integers do, two at a time
  uint32_t pairs = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
  pairs = __vmaxu2(pairs, __shfl_xor_sync(mask, pairs, 1));
  pairs = __vmaxu2(pairs, __shfl_xor_sync(mask, pairs, 2));
  const int s = scale_code<FMT>(max(pairs & 0xffffu, pairs >> 16));
  // times 2^(127 - s), in bf16: exact, but for products below 2^-126, which are zeros of the element type anyway
  const uint32_t inv = pair((uint32_t)(254 - s) << 7);
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t y = mul_bf16x2(w[i], inv);
    v[2 * i] = bf16_lo(y);
    v[2 * i + 1] = bf16_hi(y);
  }
  constexpr int kLast = FMT == kCacheMx8 ? 247 : 253;      // the largest numbers' scale: what would round to 2^128 is rounded toward zero
  if (s >= kLast) {
    // (infinities and NaN, s = 255: zeros)
    constexpr float most = FMT == kCacheMx8 ? 240.f : 3.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = s == 255 ? 0.f : fminf(fmaxf(v[i], -most), most);
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

// A CTA takes kWriteRows x 4096 / D consecutive tokens of one head, so that it writes whole sectors of scales, and a thread has all its rows in
// flight at once.
constexpr int kWriteRows = 1;

template <int FMT, int D>
__global__ void __launch_bounds__(256)
k_cache_write(const CacheDims dm, const uint16_t* K_new, const uint16_t* V_new,
              const int32_t* cu_q, const int32_t* seq_lens, const int32_t* table,
              uint8_t* K, uint8_t* V, uint8_t* K_scale, uint8_t* V_scale,
              int32_t* status_word) {
  constexpr int CH = D / 16, kRows = 256 / CH;  // threads of a row, rows of one access of the CTA
  const int blk = dm.by_Hkv(blockIdx.x), h = blockIdx.x - blk * dm.Hkv;
  const int t0 = blk * (kRows * kWriteRows) + threadIdx.x / CH, c = threadIdx.x % CH;
  pdl_wait();
  pdl_launch_dependents();
  uint4 k[kWriteRows][2], v[kWriteRows][2];
#pragma unroll
  for (int u = 0; u < kWriteRows; ++u) {
    const int64_t t = t0 + u * kRows;
    const uint16_t* const kr = K_new + t * dm.kns[0] + h * dm.kns[1] + c * 8;
    const uint16_t* const vr = V_new + t * dm.vns[0] + h * dm.vns[1] + c * 8;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      k[u][i] = v[u][i] = make_uint4(0, 0, 0, 0);
      if (t < dm.n_tokens && K_new) k[u][i] = __ldcs(reinterpret_cast<const uint4*>(kr + i * (D / 2)));
      if (t < dm.n_tokens && V_new) v[u][i] = __ldcs(reinterpret_cast<const uint4*>(vr + i * (D / 2)));
    }
  }
  int lo = find_seq(cu_q, dm.n_seq, t0 - (int)(threadIdx.x & 31) / CH);      // of the warp's first row
  bool bad = false;
  int page[kWriteRows], r[kWriteRows];
  CacheSeq s = cache_seq(dm, cu_q, seq_lens, lo);
#pragma unroll
  for (int u = 0; u < kWriteRows; ++u) {
    const int t = t0 + u * kRows;
    page[u] = -1;
    r[u] = 0;
    if (t >= dm.n_tokens) continue;
    while (lo + 1 < dm.n_seq && cu_q[lo + 1] <= t) s = cache_seq(dm, cu_q, seq_lens, ++lo);
    bad = bad || s.bad;
    const int pos = s.len - s.n_all + (t - s.q0);
    if (t < s.q0 || t - s.q0 >= s.n || pos < 0 || pos >= dm.max_keys) continue;
    const int e = dm.by_page(pos);
    r[u] = pos - e * dm.page;
    page[u] = table[lo * dm.table_stride + e];
    if (page[u] < 0 || page[u] >= dm.n_pages) { bad = true; page[u] = -1; }
  }
  constexpr int kUnit = FMT == kCacheBf16 ? 2 : 1;
#pragma unroll
  for (int u = 0; u < kWriteRows; ++u) {
    const bool here = page[u] >= 0;              // (the threads of a row agree)
    const unsigned mask = __ballot_sync(0xffffffffu, here);
    if (here) {
      const int64_t srow = (((int64_t)page[u] * dm.Hkv + h) * dm.page + r[u]) * (D / 32);
      uint8_t* const kr = K + (page[u] * dm.ks[0] + h * dm.ks[1] + r[u] * dm.ks[2]) * kUnit;
      uint8_t* const vr = V + (page[u] * dm.vs[0] + h * dm.vs[1] + r[u] * dm.vs[2]) * kUnit;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (K_new) put8<FMT>(k[u][i], kr, K_scale + srow, c + i * CH, mask);
        if (V_new) put8<FMT>(v[u][i], vr, V_scale + srow, c + i * CH, mask);
      }
    }
    __syncwarp();
  }
  if (bad && c == 0) cache_status(status_word, HGA_STATUS_BAD_INDEX);
}

// Eight numbers of a row out of the cache
template <int FMT> struct Raw8 { typedef uint4 type; };
template <> struct Raw8<kCacheMx8> { typedef uint2 type; };
template <> struct Raw8<kCacheMx4> { typedef uint32_t type; };

__device__ __forceinline__ uint4 take8(uint4 x, uint32_t) { return x; }
// fp16 pairs, each an element's value, as bf16 times 2^(scale - 127).  fp16's sign, exponent and mantissa moved to where bf16 has them are the
// number times 2^-112.
__device__ __forceinline__ uint4 scaled(const uint32_t (&x)[4], uint32_t scale) {
  // (2^(scale - 127 + 112) is beyond bf16 from 143 on; 255 is NaN)
  const uint32_t first = pair(scale <= 142 ? (scale + 112) << 7 : (127 + 112) << 7);
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = mul_bf16x2((x[i] & 0x80008000u) | ((x[i] >> 3) & 0x0fff0fffu), first);
  if (scale > 142) {
    const uint32_t rest = pair(scale_bits(scale));
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = mul_bf16x2(y[i], rest);
  }
  return make_uint4(y[0], y[1], y[2], y[3]);
}
__device__ __forceinline__ uint4 take8(uint2 x, uint32_t scale) {
  uint32_t y[4];
  e4m3x4_to_f16(x.x, y[0], y[1]);
  e4m3x4_to_f16(x.y, y[2], y[3]);
  uint4 r = scaled(y, scale);
  const uint32_t n0 = e4m3_nan(x.x), n1 = e4m3_nan(x.y);
  if (n0 | n1) {      // (fp16's NaN is a finite number where its bits are moved; hga_cache_write makes none)
    r.x |= nan_halves(n0, false); r.y |= nan_halves(n0, true);
    r.z |= nan_halves(n1, false); r.w |= nan_halves(n1, true);
  }
  return r;
}
__device__ __forceinline__ uint4 take8(uint32_t x, uint32_t scale) {
  uint32_t y[4];
  e2m1x8_to_f16(x, y[0], y[1], y[2], y[3]);
  return scaled(y, scale);
}

constexpr int kReadRows = 2;      // rows a thread has in flight

template <int FMT, int D>
__global__ void __launch_bounds__(256)
k_cache_read(const CacheDims dm, int tok_begin, int n, const int32_t* seq_lens, const int32_t* table,
             const uint8_t* K, const uint8_t* V, const uint8_t* K_scale,
             const uint8_t* V_scale, uint16_t* K_out, uint16_t* V_out, int32_t* status_word,
             int blocks_per_head) {
  typedef typename Raw8<FMT>::type Raw;
  typedef typename ScaleWord<D>::type SW;
  constexpr int CH = D / 16, kRows = 256 / CH;
  const int bh = blockIdx.x / blocks_per_head, blk = blockIdx.x - bh * blocks_per_head;
  const int i = dm.by_Hkv(bh), h = bh - i * dm.Hkv;
  const int c = threadIdx.x % CH, r0 = blk * (kRows * kReadRows) + threadIdx.x / CH;
  constexpr int kUnit = FMT == kCacheBf16 ? 2 : 1;
  pdl_wait();
  pdl_launch_dependents();
  const int len = seq_lens[i];
  bool bad = len < 0 || len > dm.max_keys;
  const int end = min(min(max(len, 0), dm.max_keys) - tok_begin, n);      // rows of this sequence that are there
  const uint8_t* const k0 = K + h * dm.ks[1] * kUnit + c * sizeof(Raw);
  const uint8_t* const v0 = V + h * dm.vs[1] * kUnit + c * sizeof(Raw);
  Raw k[kReadRows][2], v[kReadRows][2];
  SW ks[kReadRows], vs[kReadRows];
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    const int r = r0 + u * kRows;
    k[u][0] = k[u][1] = v[u][0] = v[u][1] = Raw{};
    ks[u] = vs[u] = 0;
    if (r < end) {
      const int pos = tok_begin + r, e = dm.by_page(pos), pr = pos - e * dm.page;
      const int page = table[i * dm.table_stride + e];
      if (page < 0 || page >= dm.n_pages) { bad = true; continue; }
      const int64_t srow = (((int64_t)page * dm.Hkv + h) * dm.page + pr) * (D / 32);
      const uint8_t* const kr = k0 + (page * dm.ks[0] + pr * dm.ks[2]) * kUnit;
      const uint8_t* const vr = v0 + (page * dm.vs[0] + pr * dm.vs[2]) * kUnit;
      if (K_out) {
#pragma unroll
        for (int j = 0; j < 2; ++j) k[u][j] = *reinterpret_cast<const Raw*>(kr + j * CH * sizeof(Raw));
        if (FMT != kCacheBf16) ks[u] = *reinterpret_cast<const SW*>(K_scale + srow);
      }
      if (V_out) {
#pragma unroll
        for (int j = 0; j < 2; ++j) v[u][j] = *reinterpret_cast<const Raw*>(vr + j * CH * sizeof(Raw));
        if (FMT != kCacheBf16) vs[u] = *reinterpret_cast<const SW*>(V_scale + srow);
      }
    }
  }
  int64_t at = i * dm.outs[0] + h * dm.outs[1] + r0 * dm.outs[2] + c * 8;
  const int sh = 8 * (c >> 2);                    // of this thread's block in the half
#pragma unroll
  for (int u = 0; u < kReadRows; ++u, at += kRows * dm.outs[2]) {
    if (r0 + u * kRows >= end) break;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int s = sh + j * 4 * (D / 32);
      if (K_out) *reinterpret_cast<uint4*>(K_out + at + j * (D / 2)) = take8(k[u][j], (ks[u] >> s) & 255u);
      if (V_out) *reinterpret_cast<uint4*>(V_out + at + j * (D / 2)) = take8(v[u][j], (vs[u] >> s) & 255u);
    }
  }
  if (bad && c == 0) cache_status(status_word, HGA_STATUS_BAD_INDEX);
}

template <int FMT, int D>
int write_of(const CacheDims& dm, const void* K_new, const void* V_new, const int32_t* cu_q, const int32_t* seq_lens,
             const int32_t* table, void* K, void* V, void* K_scale, void* V_scale, int32_t* status_word, cudaStream_t st) {
  constexpr int per = 256 / (D / 16) * kWriteRows;
  PdlLaunch cfg(dim3((unsigned)((int64_t)((dm.n_tokens + per - 1) / per) * dm.Hkv)), 256, 0, st, 0);
  const cudaError_t e = cudaLaunchKernelEx(&cfg.c, k_cache_write<FMT, D>, dm, (const uint16_t*)K_new, (const uint16_t*)V_new, cu_q,
                                           seq_lens, table, (uint8_t*)K, (uint8_t*)V, (uint8_t*)K_scale, (uint8_t*)V_scale,
                                           status_word);
  count_launch(HGA_KERNELS_CACHE);
  return record_cuda(e);
}

template <int FMT, int D>
int read_of(const CacheDims& dm, int tok_begin, int n, const int32_t* seq_lens, const int32_t* table, const void* K, const void* V,
            const void* K_scale, const void* V_scale, void* K_out, void* V_out, int32_t* status_word, cudaStream_t st) {
  constexpr int per = 256 / (D / 16) * kReadRows;
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
