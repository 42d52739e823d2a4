// C-ABI entry points of the paged key/value cache: argument validation, stride resolution, dispatch.
#include <algorithm>
#include <cmath>

#include "hga_cache.cuh"

namespace hga {

static bool misaligned(const void* p, unsigned bytes = 16) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// Strides of a tensor, dense where all are zero.  unit: elements that make 16 bytes; row: elements of the innermost axis.
template <int N>
static int take_strides(const int64_t (&in)[N], int64_t (&out)[N], const int64_t (&dense)[N], int unit, int row) {
  bool none = true;
  for (int i = 0; i < N; ++i) none = none && in[i] == 0;
  for (int i = 0; i < N; ++i) {
    out[i] = none ? dense[i] : in[i];
    if (out[i] < 0 || out[i] % unit) return HGA_ERR_ALIGN;
  }
  // rows that overlap: the innermost two axes of every tensor here hold rows side by side
  if (out[N - 1] < row && out[N - 1] != 0) return HGA_ERR_SHAPE;
  return HGA_OK;
}

static int resolve_cache(const hga_cache_params* p, CacheDims& dm) {
  if (!p) return HGA_ERR_NULL;
  if (p->n_seq < 1 || p->n_seq > 65535 || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads) return HGA_ERR_SHAPE;
  if (p->head_dim != 64 && p->head_dim != 128) return HGA_ERR_UNSUPPORTED;
  if (p->n_q_heads / p->n_kv_heads > 128) return HGA_ERR_UNSUPPORTED;
  if (p->format != HGA_CACHE_BF16 && p->format != HGA_CACHE_MXFP8 && p->format != HGA_CACHE_MXFP4) return HGA_ERR_UNSUPPORTED;
  if (p->flags != 0 || p->reserved != 0) return HGA_ERR_UNSUPPORTED;
  if (p->page_size < 8 || p->page_size > 4096 || p->page_size % 8) return HGA_ERR_SHAPE;
  if (p->n_pages < 1 || p->max_pages < 1 || (int64_t)p->max_pages * p->page_size > 0x7fffff00) return HGA_ERR_SHAPE;
  if (p->n_tokens < 0 || p->max_new < 1 || p->max_len < 0) return HGA_ERR_SHAPE;
  // rows of the packed tensors, and of all new tokens of one sequence, are counted in 32 bits
  if ((int64_t)p->n_tokens * p->n_q_heads > 0x7fffff00 || (int64_t)p->n_seq * p->n_kv_heads > 0x7fffff00) return HGA_ERR_SHAPE;
  dm.n_seq = p->n_seq; dm.Hq = p->n_q_heads; dm.Hkv = p->n_kv_heads; dm.G = dm.Hq / dm.Hkv; dm.d = p->head_dim;
  dm.page = p->page_size; dm.n_pages = p->n_pages; dm.max_pages = p->max_pages; dm.format = p->format;
  dm.n_tokens = p->n_tokens;
  dm.max_new = std::min(p->max_new, std::max(p->n_tokens, 1));
  dm.max_keys = p->max_pages * p->page_size;
  if (p->max_len > 0) dm.max_keys = std::min(dm.max_keys, p->max_len);
  if (dm.max_keys > 1 << 30) return HGA_ERR_SHAPE;      // (a position and the keys of a part behind it are an int)
  dm.scale = p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)dm.d);
  if (p->table_stride != 0 && p->table_stride < p->max_pages) return HGA_ERR_SHAPE;
  dm.table_stride = p->table_stride ? p->table_stride : p->max_pages;
  const int64_t d = dm.d, row = dm.format == HGA_CACHE_BF16 ? d : cache_row_bytes(dm.format, dm.d);
  const int64_t q[2] = {dm.Hq * d, d}, kv[2] = {dm.Hkv * d, d};
  const int64_t pool[3] = {dm.Hkv * (int64_t)dm.page * row, dm.page * row, row};
  const int unit = dm.format == HGA_CACHE_BF16 ? 8 : 16;
  int rc;
  if ((rc = take_strides(p->q_stride, dm.qs, q, 8, dm.d)) || (rc = take_strides(p->o_stride, dm.os, q, 8, dm.d)) ||
      (rc = take_strides(p->kn_stride, dm.kns, kv, 8, dm.d)) || (rc = take_strides(p->vn_stride, dm.vns, kv, 8, dm.d)) ||
      (rc = take_strides(p->k_stride, dm.ks, pool, unit, (int)row)) || (rc = take_strides(p->v_stride, dm.vs, pool, unit, (int)row)))
    return rc;
  if (dm.os[0] == 0 || dm.os[1] == 0 || dm.ks[2] == 0 || dm.vs[2] == 0) return HGA_ERR_SHAPE;
  // (a tensor map's strides: positive, below 2^40 bytes)
  const int64_t most = ((int64_t)1 << 40) / (dm.format == HGA_CACHE_BF16 ? 2 : 1);
  for (int i = 0; i < 2; ++i) {
    if ((i ? dm.Hkv : dm.n_pages) == 1) dm.ks[i] = dm.vs[i] = 16;      // (of no consequence)
    if (dm.ks[i] < 16 || dm.vs[i] < 16 || dm.ks[i] >= most || dm.vs[i] >= most) return HGA_ERR_SHAPE;
  }
  if (dm.ks[2] >= most || dm.vs[2] >= most) return HGA_ERR_SHAPE;
  dm.by_page = Div(dm.page); dm.by_Hkv = Div(dm.Hkv); dm.by_G = Div(dm.G);
  return HGA_OK;
}

// Which kernel: rows of a sequence's (new tokens x query heads of a group) in tiles of 16 that each read the keys again, or in tiles of 128.
// 16 sequences of up to 32K, 4 key/value heads, us (tiles of 16 / 128): bf16 35 rows 137 / 147, 63 rows 241 / 152; e2m1 35 rows 106 / 235, 63
// rows 173 / 238, 126 rows - / 235 (converting the keys is most of the work there).
static bool few_rows(const CacheDims& dm) { return (int64_t)dm.max_new * dm.G <= (dm.format == HGA_CACHE_BF16 ? 48 : 64); }
static CacheSplit attn_split(const CacheDims& dm) { return few_rows(dm) ? cache_rows_split(dm) : cache_tensor_split(dm); }

}  // namespace hga

using namespace hga;

extern "C" {

int hga_cache_workspace_bytes(const hga_cache_params* p, size_t* bytes) {
  CacheDims dm;
  const int rc = resolve_cache(p, dm);
  if (rc) return rc;
  if (!bytes) return HGA_ERR_NULL;
  *bytes = attn_split(dm).bytes(dm);
  return HGA_OK;
}

int hga_cache_write(const hga_cache_params* p, const void* K_new, const void* V_new, const int32_t* cu_q, const int32_t* seq_lens,
                    const int32_t* block_table, void* K_cache, void* V_cache, void* K_scale, void* V_scale, int32_t* status_word,
                    void* stream) {
  CacheDims dm;
  const int rc = resolve_cache(p, dm);
  if (rc) return rc;
  const bool scaled = dm.format != HGA_CACHE_BF16;
  if ((dm.n_tokens > 0 && !K_new && !V_new) || !cu_q || !seq_lens || !block_table) return HGA_ERR_NULL;      // (a tensor of no rows may have no address)
  if ((K_new && (!K_cache || (scaled && !K_scale))) || (V_new && (!V_cache || (scaled && !V_scale)))) return HGA_ERR_NULL;
  if (misaligned(K_new) || misaligned(V_new) || misaligned(K_cache) || misaligned(V_cache) || misaligned(K_scale) || misaligned(V_scale) ||
      misaligned(cu_q, 4) || misaligned(seq_lens, 4) || misaligned(block_table, 4) || misaligned(status_word, 4))
    return HGA_ERR_ALIGN;
  if (dm.n_tokens == 0) return HGA_OK;
  return launch_cache_write(dm, K_new, V_new, cu_q, seq_lens, block_table, K_cache, V_cache, K_scale, V_scale, status_word,
                            (cudaStream_t)stream);
}

int hga_cache_read(const hga_cache_params* p, int32_t tok_begin, int32_t tok_end, const int32_t* seq_lens, const int32_t* block_table,
                   const void* K_cache, const void* V_cache, const void* K_scale, const void* V_scale, void* K_out, void* V_out,
                   int32_t* status_word, void* stream) {
  CacheDims dm;
  int rc = resolve_cache(p, dm);
  if (rc) return rc;
  const bool scaled = dm.format != HGA_CACHE_BF16;
  if ((tok_end > tok_begin && !K_out && !V_out) || !seq_lens || !block_table) return HGA_ERR_NULL;
  if ((K_out && (!K_cache || (scaled && !K_scale))) || (V_out && (!V_cache || (scaled && !V_scale)))) return HGA_ERR_NULL;
  if (misaligned(K_out) || misaligned(V_out) || misaligned(K_cache) || misaligned(V_cache) || misaligned(K_scale) || misaligned(V_scale) ||
      misaligned(seq_lens, 4) || misaligned(block_table, 4) || misaligned(status_word, 4))
    return HGA_ERR_ALIGN;
  if (tok_begin < 0 || tok_end < tok_begin || tok_end > 0x7fffff00) return HGA_ERR_SHAPE;      // (rows of the last CTA are counted in an int)
  const int64_t n = tok_end - tok_begin, d = dm.d, dense[3] = {dm.Hkv * n * d, n * d, d};
  if ((rc = take_strides(p->out_stride, dm.outs, dense, 8, dm.d))) return rc;
  if (n > 0 && dm.outs[2] == 0) return HGA_ERR_SHAPE;
  if (n == 0) return HGA_OK;
  if ((n + 31) / 32 * dm.n_seq * dm.Hkv > 0x7fffffff) return HGA_ERR_SHAPE;      // (a CTA has more than 32 rows)
  return launch_cache_read(dm, tok_begin, tok_end, seq_lens, block_table, K_cache, V_cache, K_scale, V_scale, K_out, V_out, status_word,
                           (cudaStream_t)stream);
}

int hga_cache_attn(const hga_cache_params* p, const void* Q, const int32_t* cu_q, const int32_t* seq_lens, const int32_t* block_table,
                   const void* K_cache, const void* V_cache, const void* K_scale, const void* V_scale, void* O, float* LSE,
                   void* workspace, size_t workspace_bytes, int32_t* status_word, void* stream) {
  CacheDims dm;
  const int rc = resolve_cache(p, dm);
  if (rc) return rc;
  if ((dm.n_tokens > 0 && (!Q || !O)) || !cu_q || !seq_lens || !block_table || !K_cache || !V_cache) return HGA_ERR_NULL;
  if (dm.format != HGA_CACHE_BF16 && (!K_scale || !V_scale)) return HGA_ERR_NULL;
  if (misaligned(Q) || misaligned(K_cache) || misaligned(V_cache) || misaligned(K_scale) || misaligned(V_scale) || misaligned(O) ||
      misaligned(LSE, 4) || misaligned(cu_q, 4) || misaligned(seq_lens, 4) || misaligned(block_table, 4) || misaligned(status_word, 4))
    return HGA_ERR_ALIGN;
  const CacheSplit sp = attn_split(dm);
  const size_t need = sp.bytes(dm);
  if (need && (!workspace || workspace_bytes < need)) return HGA_ERR_WORKSPACE;
  if (misaligned(workspace)) return HGA_ERR_ALIGN;
  if (dm.n_tokens == 0) return HGA_OK;
  if (!few_rows(dm))
    return launch_cache_attn_sm100(dm, Q, cu_q, seq_lens, block_table, K_cache, V_cache, K_scale, V_scale, O, LSE, workspace, status_word,
                                   (cudaStream_t)stream);
  return launch_cache_attn_rows(dm, sp, Q, cu_q, seq_lens, block_table, K_cache, V_cache, K_scale, V_scale, O, LSE, workspace, status_word,
                                (cudaStream_t)stream);
}

}  // extern "C"
