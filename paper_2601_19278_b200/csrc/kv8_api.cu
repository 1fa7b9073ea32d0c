// C entry points of the paged 8-bit KV cache: argument checks and launches.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "../../include/dart.h"
#include "kv8.cuh"

using namespace dart;

namespace {

bool aligned16(const void* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool null_or_aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int fail(cudaError_t e) {
  record_global_cuda_error(e);
  return DART_ERR_CUDA;
}

bool page_tokens_ok(int pt) { return pt == 16 || pt == 32 || pt == 64 || pt == 128; }
bool table_ok(int max_seqs, int max_pages, int pt) {
  return max_seqs >= 1 && max_seqs <= 65536 && max_pages >= 1 && (long long)max_pages * pt < (1ll << 31) - (1 << 21);
}

bool cache_shape_ok(const dart_kv8_cache* c) {
  return c != nullptr && (c->format == DART_KV8_E4M3 || c->format == DART_KV8_INT8) && c->n_layers >= 1 && c->n_layers <= 1024 && c->n_pages >= 1 &&
         c->n_pages <= (1 << 24) && c->n_kv_heads >= 1 && c->n_kv_heads <= 256 && page_tokens_ok(c->page_tokens) &&
         (c->head_dim == 64 || c->head_dim == 128);
}
bool cache_ok(const dart_kv8_cache* c) {
  return cache_shape_ok(c) && aligned16(c->k_pages) && aligned16(c->v_pages) && aligned4(c->k_scale) && aligned4(c->v_scale);
}

bool attn_shape_ok(const dart_kv8_cache* c, int batch, int rows, int n_q_heads, int max_len) {
  return cache_shape_ok(c) && batch >= 1 && batch <= 1024 && rows >= 1 && rows <= 4096 && n_q_heads >= 1 && n_q_heads % c->n_kv_heads == 0 &&
         n_q_heads / c->n_kv_heads <= 128 && max_len >= 0;
}

Kv8AttnArgs attn_shape(const dart_kv8_cache* c, int batch, int rows, int n_q_heads, int max_len) {
  Kv8AttnArgs a;
  memset(&a, 0, sizeof(a));
  a.c.format = c->format; a.c.n_pages = c->n_pages; a.c.hkv = c->n_kv_heads; a.c.pt = c->page_tokens; a.c.dh = c->head_dim;
  a.c.pt_log2 = c->page_tokens == 16 ? 4 : c->page_tokens == 32 ? 5 : c->page_tokens == 64 ? 6 : 7;
  a.batch = batch; a.rows = rows; a.hq = n_q_heads; a.G = n_q_heads / c->n_kv_heads; a.max_len = max_len;
  a.scale_log2e = (float)(1.4426950408889634 / sqrt((double)c->head_dim));
  return a;
}

// The same with a window; positions lie below max_len + rows, so a wider window or more sinks than that are no more (and sums with
// them stay in 32 bits).
Kv8AttnArgs window_shape(Kv8AttnArgs a, int window, int sinks) {
  const long long all = (long long)a.max_len + a.rows;
  a.window = (int)std::min<long long>(window, all);
  a.sinks = (int)std::min<long long>(sinks, all);
  return a;
}

dart_kv8_plan plan_of(Kv8AttnArgs a, int with_new_rows) {
  static const bf16 some_row{};
  if (with_new_rows) a.k_new = &some_row;      // (never read)
  const Kv8Plan p = kv8_attention_plan(a);
  return dart_kv8_plan{p.umma, p.umma ? p.n_tiles : 0, p.paired, p.umma ? p.chunk * 128 : p.chunk, p.max_chunks};
}

bool pages_ok(const dart_kv8_pages* p) {
  return p != nullptr && p->n_pages >= 1 && p->n_pages <= (1 << 24) && page_tokens_ok(p->page_tokens) &&
         table_ok(p->max_seqs, p->max_pages, p->page_tokens) && aligned4(p->page_table) && aligned4(p->seq_lens) && aligned4(p->ref_count);
}
Kv8PagesArgs pages_args(const dart_kv8_pages* p) {
  return Kv8PagesArgs{p->n_pages, p->page_tokens, p->max_seqs, p->max_pages, p->page_table, p->seq_lens, p->ref_count};
}
Kv8PoolArgs pool_args(const dart_kv8_cache* c) {
  return Kv8PoolArgs{static_cast<uint8_t*>(c->k_pages), static_cast<uint8_t*>(c->v_pages), c->k_scale, c->v_scale, c->n_layers, c->n_pages,
                     c->n_kv_heads, (long long)c->n_kv_heads * c->page_tokens * c->head_dim};
}
bool list_ok(const int32_t* l, int n) { return n >= 1 && n <= 1024 && aligned4(l); }

}  // namespace

extern "C" {

size_t dart_kv8_attention_workspace_bytes(const dart_kv8_cache* cache, int32_t batch, int32_t rows, int32_t n_q_heads, int32_t max_len) {
  if (!attn_shape_ok(cache, batch, rows, n_q_heads, max_len)) return 0;
  return kv8_attention_workspace(attn_shape(cache, batch, rows, n_q_heads, max_len));
}

int dart_kv8_attention_plan(const dart_kv8_cache* cache, int32_t batch, int32_t rows, int32_t n_q_heads, int32_t max_len, int32_t with_new_rows,
                            dart_kv8_plan* out) {
  if (out == nullptr || !attn_shape_ok(cache, batch, rows, n_q_heads, max_len)) return DART_ERR_INVALID_ARG;
  *out = plan_of(attn_shape(cache, batch, rows, n_q_heads, max_len), with_new_rows);
  return DART_OK;
}

size_t dart_kv8_attention_window_workspace_bytes(const dart_kv8_cache* cache, int32_t batch, int32_t rows, int32_t n_q_heads, int32_t max_len,
                                                 int32_t window, int32_t sinks) {
  if (!attn_shape_ok(cache, batch, rows, n_q_heads, max_len) || window < 1 || sinks < 0) return 0;
  return kv8_attention_workspace(window_shape(attn_shape(cache, batch, rows, n_q_heads, max_len), window, sinks));
}

int dart_kv8_attention_window_plan(const dart_kv8_cache* cache, int32_t batch, int32_t rows, int32_t n_q_heads, int32_t max_len, int32_t window,
                                   int32_t sinks, int32_t with_new_rows, dart_kv8_plan* out) {
  if (out == nullptr || !attn_shape_ok(cache, batch, rows, n_q_heads, max_len) || window < 1 || sinks < 0) return DART_ERR_INVALID_ARG;
  *out = plan_of(window_shape(attn_shape(cache, batch, rows, n_q_heads, max_len), window, sinks), with_new_rows);
  return DART_OK;
}

static int attention(const dart_kv8_cache* cache, const dart_kv8_attn_in* in, const dart_kv8_window* w, bool selftest, int spin, int withhold,
                     void* cuda_stream) {
  if (in == nullptr || !cache_ok(cache) || !attn_shape_ok(cache, in->batch, in->rows, in->n_q_heads, in->max_len)) return DART_ERR_INVALID_ARG;
  const int pt = cache->page_tokens, dh = cache->head_dim;
  if (in->layer < 0 || in->layer >= cache->n_layers || !table_ok(in->max_seqs, in->max_pages, pt)) return DART_ERR_INVALID_ARG;
  if (in->max_len > (long long)in->max_pages * pt || (in->slots == nullptr && in->batch > in->max_seqs)) return DART_ERR_INVALID_ARG;
  if (!aligned16(in->q) || !aligned16(in->out) || in->q_stride < (int64_t)in->n_q_heads * dh || in->q_stride % 8 != 0) return DART_ERR_INVALID_ARG;
  if ((in->k_new == nullptr) != (in->v_new == nullptr)) return DART_ERR_INVALID_ARG;
  if (in->k_new != nullptr && (!aligned16(in->k_new) || !aligned16(in->v_new) || in->new_stride < (int64_t)cache->n_kv_heads * dh ||
                               in->new_stride % 8 != 0))
    return DART_ERR_INVALID_ARG;
  if (in->mask != nullptr && (in->k_new == nullptr || in->rows > 64)) return DART_ERR_INVALID_ARG;
  if (!aligned4(in->seq_lens) || !aligned4(in->page_table) || !null_or_aligned4(in->slots) || !null_or_aligned4(in->n_rows) ||
      !null_or_aligned4(in->status))
    return DART_ERR_INVALID_ARG;
  Kv8AttnArgs a = attn_shape(cache, in->batch, in->rows, in->n_q_heads, in->max_len);
  if (w != nullptr) {
    if (w->window < 1 || w->sinks < 0 || (w->positions == nullptr) != (in->mask == nullptr) || !null_or_aligned4(w->positions)) return DART_ERR_INVALID_ARG;
    a = window_shape(a, w->window, w->sinks);
    a.positions = w->positions;
  }
  if (!aligned16(in->workspace) || in->workspace_bytes < kv8_attention_workspace(a)) return DART_ERR_INVALID_ARG;
  if (selftest && !kv8_attention_plan(a).umma) return DART_ERR_INVALID_ARG;
  const int arch = check_sm100();
  if (arch != DART_OK) return arch;
  const size_t layer = (size_t)in->layer * cache->n_pages * cache->n_kv_heads;
  a.c.k = static_cast<const uint8_t*>(cache->k_pages) + layer * pt * dh;
  a.c.v = static_cast<const uint8_t*>(cache->v_pages) + layer * pt * dh;
  a.c.ks = cache->k_scale + layer;
  a.c.vs = cache->v_scale + layer;
  a.max_seqs = in->max_seqs; a.max_pages = in->max_pages;
  a.q_stride = in->q_stride; a.new_stride = in->new_stride;
  a.q = static_cast<const bf16*>(in->q); a.k_new = static_cast<const bf16*>(in->k_new); a.v_new = static_cast<const bf16*>(in->v_new);
  a.slots = in->slots; a.seq_lens = in->seq_lens; a.table = in->page_table; a.n_rows = in->n_rows; a.mask = in->mask;
  a.out = static_cast<bf16*>(in->out); a.status = in->status;
  const cudaError_t e = launch_kv8_attention(a, in->workspace, spin, withhold, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? DART_OK : fail(e);
}

int dart_kv8_attention(const dart_kv8_cache* cache, const dart_kv8_attn_in* in, void* cuda_stream) {
  return attention(cache, in, nullptr, false, kKv8Spin, -1, cuda_stream);
}

int dart_kv8_attention_window(const dart_kv8_cache* cache, const dart_kv8_attn_in* in, const dart_kv8_window* window, void* cuda_stream) {
  if (window == nullptr) return DART_ERR_INVALID_ARG;
  return attention(cache, in, window, false, kKv8Spin, -1, cuda_stream);
}

static int selftest(const dart_kv8_cache* cache, const dart_kv8_attn_in* in, const dart_kv8_window* w, int spin_limit, int missing_from, void* cuda_stream) {
  if (in == nullptr || in->status == nullptr || spin_limit < 1 || spin_limit > 100000 || missing_from < 0) return DART_ERR_INVALID_ARG;
  return attention(cache, in, w, true, spin_limit, missing_from, cuda_stream);
}

int dart_selftest_kv8_wait(const dart_kv8_cache* cache, const dart_kv8_attn_in* in, int32_t spin_limit, int32_t missing_from, void* cuda_stream) {
  return selftest(cache, in, nullptr, spin_limit, missing_from, cuda_stream);
}

int dart_selftest_kv8_window_wait(const dart_kv8_cache* cache, const dart_kv8_attn_in* in, const dart_kv8_window* window, int32_t spin_limit,
                                  int32_t missing_from, void* cuda_stream) {
  if (window == nullptr) return DART_ERR_INVALID_ARG;
  return selftest(cache, in, window, spin_limit, missing_from, cuda_stream);
}

static int append(const dart_kv8_cache* cache, const dart_kv8_append_in* in, const int32_t* ref, void* cuda_stream) {
  if (in == nullptr || !cache_ok(cache)) return DART_ERR_INVALID_ARG;
  const int pt = cache->page_tokens, dh = cache->head_dim;
  if (in->first_layer < 0 || in->n_layers < 1 || in->first_layer > cache->n_layers - in->n_layers || in->batch < 1 || in->batch > 1024 ||
      in->rows < 1 || in->rows > (1 << 20) || in->max_append < 1 || in->max_append > (1 << 20) ||
      (in->row_index == nullptr && in->max_append > in->rows) || !table_ok(in->max_seqs, in->max_pages, pt) ||
      (in->slots == nullptr && in->batch > in->max_seqs))
    return DART_ERR_INVALID_ARG;
  if (!aligned16(in->k_new) || !aligned16(in->v_new) || in->row_stride < (int64_t)cache->n_kv_heads * dh || in->row_stride % 8 != 0 ||
      in->layer_stride % 8 != 0 || in->layer_stride < 0)
    return DART_ERR_INVALID_ARG;
  if (!aligned4(in->seq_lens) || !aligned4(in->page_table) || !null_or_aligned4(in->slots) || !null_or_aligned4(in->n_append) ||
      !null_or_aligned4(in->row_index) || !null_or_aligned4(in->status))
    return DART_ERR_INVALID_ARG;
  const int arch = check_sm100();
  if (arch != DART_OK) return arch;
  Kv8AppendArgs a;
  const size_t layer = (size_t)in->first_layer * cache->n_pages * cache->n_kv_heads;
  a.k = static_cast<uint8_t*>(cache->k_pages) + layer * pt * dh;
  a.v = static_cast<uint8_t*>(cache->v_pages) + layer * pt * dh;
  a.ks = cache->k_scale + layer;
  a.vs = cache->v_scale + layer;
  a.format = cache->format; a.n_pages = cache->n_pages; a.hkv = cache->n_kv_heads; a.pt = pt; a.dh = dh;
  a.n_layers = in->n_layers; a.batch = in->batch; a.rows = in->rows; a.max_append = in->max_append;
  a.max_seqs = in->max_seqs; a.max_pages = in->max_pages;
  a.windows = (in->max_append + pt - 2) / pt + 1;      // pages that max_append rows can touch
  a.row_stride = in->row_stride; a.layer_stride = in->layer_stride;
  a.k_new = static_cast<const bf16*>(in->k_new); a.v_new = static_cast<const bf16*>(in->v_new);
  a.slots = in->slots; a.seq_lens = in->seq_lens; a.table = in->page_table; a.n_append = in->n_append; a.row_index = in->row_index;
  a.ref = ref;
  a.status = in->status;
  const cudaError_t e = launch_kv8_append(a, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? DART_OK : fail(e);
}

int dart_kv8_append(const dart_kv8_cache* cache, const dart_kv8_append_in* in, void* cuda_stream) {
  return append(cache, in, nullptr, cuda_stream);
}

int dart_kv8_append_owned(const dart_kv8_cache* cache, const dart_kv8_pages* pages, const dart_kv8_append_in* in, void* cuda_stream) {
  if (!pages_ok(pages) || !cache_ok(cache) || in == nullptr || cache->n_pages != pages->n_pages || cache->page_tokens != pages->page_tokens ||
      in->max_seqs != pages->max_seqs || in->max_pages != pages->max_pages || in->page_table != pages->page_table)
    return DART_ERR_INVALID_ARG;
  return append(cache, in, pages->ref_count, cuda_stream);
}

size_t dart_kv8_pages_workspace_bytes(const dart_kv8_pages* pages) {
  return pages != nullptr && pages->n_pages >= 1 && pages->n_pages <= (1 << 24) ? kv8_pages_workspace(pages->n_pages) : 0;
}

int dart_kv8_fork(const dart_kv8_pages* pages, const int32_t* src, const int32_t* dst, int32_t n, int32_t* status, void* cuda_stream) {
  if (!pages_ok(pages) || !list_ok(src, n) || !list_ok(dst, n) || !null_or_aligned4(status)) return DART_ERR_INVALID_ARG;
  const int arch = check_sm100();
  if (arch != DART_OK) return arch;
  const cudaError_t e = launch_kv8_fork(pages_args(pages), src, dst, n, status, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? DART_OK : fail(e);
}

int dart_kv8_release(const dart_kv8_pages* pages, const int32_t* seqs, int32_t n, int32_t* status, void* cuda_stream) {
  if (!pages_ok(pages) || !list_ok(seqs, n) || !null_or_aligned4(status)) return DART_ERR_INVALID_ARG;
  const int arch = check_sm100();
  if (arch != DART_OK) return arch;
  const cudaError_t e = launch_kv8_release(pages_args(pages), seqs, n, status, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? DART_OK : fail(e);
}

int dart_kv8_trim(const dart_kv8_pages* pages, const int32_t* seqs, int32_t n, int32_t window, int32_t sinks, int32_t* status, void* cuda_stream) {
  if (!pages_ok(pages) || !list_ok(seqs, n) || window < 1 || sinks < 0 || !null_or_aligned4(status)) return DART_ERR_INVALID_ARG;
  const int arch = check_sm100();
  if (arch != DART_OK) return arch;
  const cudaError_t e = launch_kv8_trim(pages_args(pages), seqs, n, window, sinks, status, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? DART_OK : fail(e);
}

int dart_kv8_reserve(const dart_kv8_pages* pages, const dart_kv8_cache* cache, const int32_t* seqs, const int32_t* n_new, int32_t n,
                     void* workspace, size_t workspace_bytes, int32_t* status, void* cuda_stream) {
  if (!pages_ok(pages) || !cache_ok(cache) || cache->n_pages != pages->n_pages || cache->page_tokens != pages->page_tokens ||
      !list_ok(seqs, n) || !list_ok(n_new, n) || !null_or_aligned4(status) || !aligned16(workspace) ||
      workspace_bytes < kv8_pages_workspace(pages->n_pages))
    return DART_ERR_INVALID_ARG;
  const int arch = check_sm100();
  if (arch != DART_OK) return arch;
  const cudaError_t e = launch_kv8_reserve(pages_args(pages), pool_args(cache), seqs, n_new, n, static_cast<int*>(workspace), status,
                                           static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? DART_OK : fail(e);
}

int dart_kv8_compact(const dart_kv8_pages* pages, const dart_kv8_cache* cache, int32_t* n_live_out, void* workspace, size_t workspace_bytes,
                     int32_t* status, void* cuda_stream) {
  if (!pages_ok(pages) || !cache_ok(cache) || cache->n_pages != pages->n_pages || cache->page_tokens != pages->page_tokens ||
      !null_or_aligned4(n_live_out) || !null_or_aligned4(status) || !aligned16(workspace) ||
      workspace_bytes < kv8_pages_workspace(pages->n_pages))
    return DART_ERR_INVALID_ARG;
  const int arch = check_sm100();
  if (arch != DART_OK) return arch;
  const cudaError_t e = launch_kv8_compact(pages_args(pages), pool_args(cache), n_live_out, static_cast<int*>(workspace), status,
                                           static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? DART_OK : fail(e);
}

}  // extern "C"
