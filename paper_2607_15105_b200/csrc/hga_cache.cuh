// Internal definitions of the paged key/value cache (hga_cache_*): the resolved problem, where a token lies, and the element formats.
#pragma once

#include "hga_common.cuh"

namespace hga {

// Resolved hga_cache_params, handed to kernels by value
struct CacheDims {
  int n_seq, Hq, Hkv, G, d;
  int page, n_pages, max_pages, format;
  int n_tokens, max_new, max_keys;      // max_keys: keys at or behind it are left out (the smaller of max_len and the table's reach)
  float scale;
  int64_t qs[2], os[2], kns[2], vns[2];      // (token, head)
  int64_t ks[3], vs[3];                      // (page, head, token): bf16 elements, or bytes
  int64_t outs[3];                           // (sequence, head, token)
  int64_t table_stride;
  Div by_page, by_Hkv, by_G;
};

// 32-bit words of `blocks` scale bytes: the head_dim/32 bytes of a row
template <int D> struct ScaleWord;
template <> struct ScaleWord<128> { typedef uint32_t type; };
template <> struct ScaleWord<64> { typedef uint16_t type; };

__device__ __forceinline__ void cache_status(int32_t* status_word, int bits) {
  if (status_word) atomicOr(status_word, bits);
}

// (The kernels' pointers are not __restrict__: what only such pointers read counts as never written, and the compiler may load it ahead of
// griddepcontrol.wait, when the call before, which writes the pool, is still at work.)

// The new tokens of sequence i and its resident length, held to the limits; `bad`: they had to be
struct CacheSeq {
  int q0, n;          // first row of the packed tensors, new tokens
  int len;            // resident tokens (position of new token t: len - n_all + t)
  int n_all;          // new tokens as cu_q says
  int keys;           // resident tokens that are looked at
  bool bad;
};
__device__ __forceinline__ CacheSeq cache_seq_of(const CacheDims& dm, int q0, int q1, int len) {
  CacheSeq s;
  s.bad = q0 < 0 || q1 < q0 || q1 > dm.n_tokens || len < 0 || len > dm.max_keys || (q1 - q0) > dm.max_new;
  s.q0 = min(max(q0, 0), dm.n_tokens);
  s.n_all = min(max(q1, s.q0), dm.n_tokens) - s.q0;
  s.n = min(s.n_all, dm.max_new);
  s.len = max(len, 0);
  s.keys = min(s.len, dm.max_keys);
  return s;
}
__device__ __forceinline__ CacheSeq cache_seq(const CacheDims& dm, const int32_t* cu_q, const int32_t* seq_lens, int i) {
  return cache_seq_of(dm, cu_q[i], cu_q[i + 1], seq_lens[i]);
}

// The sequence of packed row t: the last one that starts at or ahead of it (0 where none does).  For a whole warp, with the same t:
// 32 entries of cu_q are looked at at a time.
__device__ __forceinline__ int find_seq(const int32_t* cu_q, int n_seq, int t) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = n_seq;                    // it is one of lo .. lo + n - 1
  while (n > 1) {
    const int step = (n + 31) >> 5, at = lo + lane * step;
    const unsigned ahead = __ballot_sync(0xffffffffu, lane == 0 || (lane * step < n && cu_q[at] <= t));
    const int last = 31 - __clz((int)ahead);      // (cu_q does not decrease)
    n = min(step, n - last * step);
    lo += last * step;
  }
  return lo;
}

// ----------------------------------------------------------------------------- element formats
// e4m3 and e2m1 numbers have at most four significant bits and the scales are powers of two, so what is held is a bf16 number and
// every conversion below is exact.

// 2^(s - 127) as bf16 bits (s = 255: NaN)
__device__ __forceinline__ uint32_t scale_bits(uint32_t s) {
  return s == 0 ? 0x0040u : s == 255 ? 0x7fc0u : s << 7;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t pair(uint32_t lo_and_hi) { return lo_and_hi | (lo_and_hi << 16); }

// Two e4m3 numbers, in the high bytes of the two halves (low bytes zero), as bf16 times 2^-120: sign kept, exponent and mantissa moved to
// where bf16 has them.  Subnormal ones too: the exponent fields are both zero.  (NaN: 480 times 2^-120, see nan_halves.)
__device__ __forceinline__ uint32_t e4m3_to_bf16_scaled(uint32_t x) {
  return (x & 0x80008000u) | ((x >> 4) & 0x07f007f0u);
}
constexpr uint32_t kTwo120 = 0x7b807b80u;      // 2^120, twice

// Four e2m1 numbers (a nibble each, in the low 16 bits of `w`) as bf16: a look-up of the high and the low byte.  r0: nibbles 0 and 1, r1: 2 and 3.
__device__ __forceinline__ void e2m1x4_to_bf16(uint32_t w, uint32_t& r0, uint32_t& r1) {
  const uint32_t sel = w & 0x7777u;
  const uint32_t hi = __byte_perm(0x3f3f3f00u, 0x40404040u, sel);      // 0, .5, 1, 1.5 | 2, 3, 4, 6
  const uint32_t lo = __byte_perm(0xc0800000u, 0xc0804000u, sel);
  r0 = __byte_perm(lo, hi, 0x5140) | ((w << 12) & 0x8000u) | ((w << 24) & 0x80000000u);
  r1 = __byte_perm(lo, hi, 0x7362) | ((w << 4) & 0x8000u) | ((w << 16) & 0x80000000u);
}

// The bytes of a word that are e4m3's NaN (0x7f, 0xff), by their top bits; and bytes 0 and 1, or 2 and 3, of these as halves of 0x7fff, which
// make a NaN of any bf16 number
__device__ __forceinline__ uint32_t e4m3_nan(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t nan_halves(uint32_t top_bits, bool upper) {
  const uint32_t h = __byte_perm(top_bits, 0, upper ? 0x3424 : 0x1404);
  return h - (h >> 15);
}

// Four e4m3 / eight e2m1 numbers of a word as fp16 pairs, the lowest first
__device__ __forceinline__ void e4m3x4_to_f16(uint32_t x, uint32_t& r0, uint32_t& r1) {
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
      : "=r"(r0), "=r"(r1) : "r"(x));
}
__device__ __forceinline__ void e2m1x8_to_f16(uint32_t x, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(x));
}

constexpr int kCacheBf16 = HGA_CACHE_BF16, kCacheMx8 = HGA_CACHE_MXFP8, kCacheMx4 = HGA_CACHE_MXFP4;
__host__ __device__ constexpr int cache_row_bytes(int fmt, int d) { return fmt == kCacheBf16 ? 2 * d : fmt == kCacheMx8 ? d : d / 2; }

int launch_cache_write(const CacheDims& dm, const void* K_new, const void* V_new, const int32_t* cu_q, const int32_t* seq_lens,
                       const int32_t* table, void* K, void* V, void* K_scale, void* V_scale, int32_t* status_word, cudaStream_t st);
int launch_cache_read(const CacheDims& dm, int tok_begin, int tok_end, const int32_t* seq_lens, const int32_t* table, const void* K,
                      const void* V, const void* K_scale, const void* V_scale, void* K_out, void* V_out, int32_t* status_word,
                      cudaStream_t st);

// How hga_cache_attn shares out a problem: `keys` consecutive keys (a multiple of 128) go to one CTA, `parts` = what the longest
// sequence has of these.  Up to eight parts (few rows) form a cluster, whose CTAs join their results through each other's shared memory;
// otherwise they leave them in the workspace, which a second kernel joins.
// With `unit` set (chunks of one sequence), only the units of `unit` tokens from number `full` on are shared out, counted from the last and
// head by head: those that would leave most SMs idle behind the whole ones.
struct CacheSplit {
  int keys, parts;
  bool cluster;
  int tokens;               // of the partial results: the first ones
  int unit, units, full;
  size_t bytes(const CacheDims& dm) const {
    return parts > 1 && !cluster ? (size_t)parts * tokens * dm.Hq * (dm.d + 4) * sizeof(float) : 0;
  }
};
CacheSplit cache_rows_split(const CacheDims& dm);
CacheSplit cache_tensor_split(const CacheDims& dm);
int launch_cache_join(const CacheDims& dm, const CacheSplit& sp, const int32_t* cu_q, const int32_t* seq_lens, const void* workspace,
                      void* O, float* LSE, cudaStream_t st);
int launch_cache_attn_sm100(const CacheDims& dm, const void* Q, const int32_t* cu_q, const int32_t* seq_lens, const int32_t* table,
                            const void* K, const void* V, const void* K_scale, const void* V_scale, void* O, float* LSE, void* workspace,
                            int32_t* status_word, cudaStream_t st);
int launch_cache_attn_rows(const CacheDims& dm, const CacheSplit& sp, const void* Q, const int32_t* cu_q, const int32_t* seq_lens,
                           const int32_t* table, const void* K, const void* V, const void* K_scale, const void* V_scale, void* O,
                           float* LSE, void* workspace, int32_t* status_word, cudaStream_t st);

}  // namespace hga
