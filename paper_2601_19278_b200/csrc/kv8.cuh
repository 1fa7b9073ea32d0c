// The target's KV cache in 8 bits, in pages (include/dart.h): what its kernels share.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"
#include "kernels.h"

namespace dart {

enum : int { KV8_E4M3 = 0, KV8_INT8 = 1 };
enum : int { KV8_BAD_ARG = -1, KV8_CAPACITY = -4 };   // status words (dart_status)

// One layer of the pool.
struct Kv8Layer {
  int format, n_pages, hkv, pt, pt_log2, dh;
  const uint8_t *k, *v;        // [n_pages][hkv][pt][dh]
  const float *ks, *vs;        // [n_pages][hkv]
};

struct Kv8AttnArgs {
  Kv8Layer c;
  int batch, rows, hq, G, max_seqs, max_pages, max_len;
  long long q_stride, new_stride;          // elements between rows; batch entries are `rows` rows apart
  const bf16 *q, *k_new, *v_new;           // k_new null: the cache alone
  const int *slots, *seq_lens, *table, *n_rows;
  const uint8_t* mask;                     // null: causal
  bf16* out;
  int* status;
  float scale_log2e;                       // log2(e) / sqrt(dh)
};

struct Kv8AppendArgs {
  uint8_t *k, *v;                          // the pool from first_layer on
  float *ks, *vs;
  int format, n_pages, hkv, pt, dh, n_layers, batch, rows, max_append, max_seqs, max_pages, windows;
  long long row_stride, layer_stride;
  const bf16 *k_new, *v_new;
  const int *slots, *seq_lens, *table, *n_append, *row_index;
  int* status;
};

struct Kv8PagesArgs {
  int n_pages, pt, max_seqs, max_pages;
  int *table, *seq_lens, *ref;
};
// The pool as the page copies see it: every layer's K and V slab of a page, and its scales.
struct Kv8PoolArgs {
  uint8_t *k, *v;
  float *ks, *vs;
  int n_layers, n_pages, hkv;
  long long slab;                          // bytes of one page of one layer: hkv * pt * dh
};

cudaError_t launch_kv8_attention(const Kv8AttnArgs& a, void* workspace, cudaStream_t st);
size_t kv8_attention_workspace(const Kv8AttnArgs& a);
cudaError_t launch_kv8_append(const Kv8AppendArgs& a, cudaStream_t st);
cudaError_t launch_kv8_fork(const Kv8PagesArgs& p, const int* src, const int* dst, int n, int* status, cudaStream_t st);
cudaError_t launch_kv8_release(const Kv8PagesArgs& p, const int* seqs, int n, int* status, cudaStream_t st);
cudaError_t launch_kv8_reserve(const Kv8PagesArgs& p, const Kv8PoolArgs& c, const int* seqs, const int* n_new, int n, int* ws, int* status,
                               cudaStream_t st);
cudaError_t launch_kv8_compact(const Kv8PagesArgs& p, const Kv8PoolArgs& c, int* n_live, int* ws, int* status, cudaStream_t st);
size_t kv8_pages_workspace(int n_pages);

__device__ __forceinline__ void kv8_report(int* status, int code) {
  if (status != nullptr) atomicExch(status, code);
}

// What batch entry b works on.  A bad slot, length or row count reads as an empty sequence and is reported by `report`.
struct Kv8Seq { int slot, len, rows; };
__device__ __forceinline__ Kv8Seq kv8_seq(const Kv8AttnArgs& a, int b, bool report) {
  Kv8Seq s;
  s.slot = a.slots != nullptr ? a.slots[b] : b;
  s.rows = a.n_rows != nullptr ? a.n_rows[b] : a.rows;
  bool bad = s.slot < 0 || s.slot >= a.max_seqs || s.rows < 0 || s.rows > a.rows;
  s.len = bad ? 0 : a.seq_lens[s.slot];
  if (s.len < 0 || s.len > a.max_len) bad = true;
  if (bad) {
    s.slot = s.len = s.rows = 0;
    if (report) kv8_report(a.status, KV8_BAD_ARG);
  }
  return s;
}
// The page of column `col`; an id out of range reads as page 0 (in bounds; the sequence's output is void) and is reported.
__device__ __forceinline__ int kv8_page(const Kv8AttnArgs& a, int slot, int col) {
  const int p = a.table[(size_t)slot * a.max_pages + col];
  if (p >= 0 && p < a.c.n_pages) return p;
  kv8_report(a.status, KV8_BAD_ARG);
  return 0;
}

}  // namespace dart
