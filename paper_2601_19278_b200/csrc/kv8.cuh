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
  const int* ref;                          // null: every page in the table is the sequence's own
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

// How a call of the attention is cut into CTAs (launch_kv8_attention).
struct Kv8Plan {
  int umma;              // rows on tcgen05 (kv8_attn_umma.cu) instead of the streaming kernel
  int chunk;             // stream: keys a CTA takes at most; umma: its 128-key steps (beside pairs, a single tile's CTA takes twice as many)
  int max_chunks;        // CTAs that may share a (batch entry, KV head, row tile)
  int n_tiles;           // umma: 128-row tiles
  int paired;            // tiles 2p and 2p + 1 go together, an odd last one alone; else every tile alone
  float *o_part, *ml_part;
  size_t bytes;          // of workspace
  int spin;              // umma: tries of a bounded wait, of up to about 1.3 us each
  int withhold;          // umma: K's copies stop at this 64-key slot of every CTA (the self-test of the waits); -1: they do not
};
constexpr int kKv8Spin = 1000000;

// A long axis in equal parts: n CTAs of `per` (keys or steps) each, the last one shorter.
struct Kv8Split { int n, per; };
__host__ __device__ inline Kv8Split kv8_split(int total, int chunk, int unit) {
  Kv8Split s;
  s.n = total > chunk ? (total + chunk - 1) / chunk : 1;
  s.per = ((total + s.n - 1) / s.n + unit - 1) / unit * unit;      // <= chunk, a multiple of unit, as chunk is
  return s;
}
__host__ __device__ inline Kv8Split kv8_split_keys(int len, int chunk) { return kv8_split(len, chunk, 128); }

cudaError_t launch_kv8_attn_umma(const Kv8AttnArgs& a, const Kv8Plan& p, cudaStream_t st);
void kv8_umma_plan(const Kv8AttnArgs& a, Kv8Plan& p);
cudaError_t launch_kv8_attention(const Kv8AttnArgs& a, void* workspace, int spin, int withhold, cudaStream_t st);
Kv8Plan kv8_attention_plan(const Kv8AttnArgs& a);
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

// The same where an earlier error says more: a page that is missing because a reserve did not fit.
__device__ __forceinline__ void kv8_report_first(int* status, int code) {
  if (status != nullptr) atomicCAS(status, 0, code);
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

// The key steps of a row tile's group: 128 cached keys each, then 128 new rows each.  A single tile's steps alternate
// between two pipelines, so its CTA takes twice as many.
struct Kv8Tiles { int first, count, cached, steps; Kv8Split split; };      // first tile and number of tiles of the group
__device__ __forceinline__ Kv8Tiles kv8_tiles(const Kv8AttnArgs& a, const Kv8Plan& plan, const Kv8Seq& s, int tile) {
  Kv8Tiles t;
  t.first = plan.paired ? tile & ~1 : tile;
  t.count = plan.paired && t.first + 1 < plan.n_tiles ? 2 : 1;
  const int Nv = s.rows * a.G, r_end = min(s.rows, ((t.first + t.count) * 128 - 1) / a.G + 1);   // rows below r_end
  const int fresh = a.k_new == nullptr ? 0 : a.mask != nullptr ? s.rows : r_end;
  t.cached = (s.len + 127) >> 7;
  t.steps = t.first * 128 < Nv ? t.cached + ((fresh + 127) >> 7) : 0;
  t.split = kv8_split(t.steps, plan.paired && t.count == 1 ? 2 * plan.chunk : plan.chunk, 1);
  return t;
}

__device__ __forceinline__ bool kv8_sees(const Kv8AttnArgs& a, int b, int r, int y) {
  return a.mask != nullptr ? a.mask[((size_t)b * a.rows + r) * a.rows + y] != 0 : y <= r;
}

// Where a softmax's weights lie in fp16.  A weight that sets the reference maximum is 2^kKv8Bias, and the maximum moves when
// a key exceeds it by 2^kKv8Rise: 2^15 is the largest weight, which leaves the small ones 2^-25 / 2^9 = 2^-34 of the
// largest as their rounding.  That has to be small: the largest may belong to a key whose value is next to nothing, and then
// thousands of small ones make the result.  (With the largest at 1, 8192 keys behind one whose weight is 2^25 times
// theirs came out as nothing.)  O carries the bias as a factor, m and l do not.  The more bias, the smaller the rise and the
// more often a row is rescaled: 16 trees of 60 rows over pages whose scales differ by 4 take 2 % more with 9 than with none, 4 % with 11.
constexpr int kKv8Bias = 9, kKv8Rise = 15 - kKv8Bias;
constexpr float kKv8Unbias = 1.f / (1 << kKv8Bias);

__device__ __forceinline__ float kv8_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^k, -126 <= k <= 127
__device__ __forceinline__ float kv8_pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }
// The exponent that brings a row whose largest finite |x| has these bf16 bits to [1, 2).  A row of zeros gets -64: its
// values do not matter, but its weight does, and must not vanish next to the others'.  Below 2^-100 rows lose precision.
__device__ __forceinline__ int kv8_row_exp(uint32_t bits) {
  return bits == 0u ? -64 : min(max((int)(bits >> 7) - 127, -100), 126);
}
// A new row's values become multiples of 2^(its exponent - kv8_lift): largest in [2^8, 2^9) or [2^6, 2^7), as a page's largest code
// is, so that a new row weighs next to cached ones as much as it contributes.  (With the largest in [1, 2) every row's
// reference moved at its first new key, 2^7 above the cached ones: prompt chunk 267 us instead of 247.)
constexpr __host__ __device__ int kv8_lift(int format) { return format == KV8_E4M3 ? 8 : 6; }
// max of `big` and the eight |x| that are finite, as bf16 bits
__device__ __forceinline__ uint32_t kv8_max_finite(uint32_t big, const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t x0 = w[q] & 0x7fffu, x1 = (w[q] >> 16) & 0x7fffu;
    big = max(big, max(x0 < 0x7f80u ? x0 : 0u, x1 < 0x7f80u ? x1 : 0u));
  }
  return big;
}
// Zeroes the values that are not finite; whether there were any.
__device__ __forceinline__ bool kv8_zero_non_finite(uint4& v) {
  uint32_t* w = &v.x;
  bool any = false;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if ((w[q] & 0x7f80u) == 0x7f80u) { w[q] &= 0xffff0000u; any = true; }
    if ((w[q] & 0x7f800000u) == 0x7f800000u) { w[q] &= 0xffffu; any = true; }
  }
  return any;
}
// Eight bf16 times a power of two, as four fp16 pairs.
__device__ __forceinline__ void kv8_bf16x8_to_half(const uint4& v, float scale, uint32_t (&f)[4]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const __half2 h = __floats2half2_rn(__uint_as_float(w[q] << 16) * scale, __uint_as_float(w[q] & 0xffff0000u) * scale);
    f[q] = *reinterpret_cast<const uint32_t*>(&h);
  }
}

// Four codes -> two fp16 pairs, exactly.
template <int FMT>
__device__ __forceinline__ void kv8_unpack4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (FMT == KV8_E4M3) {
    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
  } else {      // 0x6400 | u is 1024 + u in fp16; u = code + 128
    const uint32_t u = w ^ 0x80808080u;
    const __half2 off = __half2half2(__ushort_as_half((unsigned short)0x6480));           // 1152
    uint32_t x = __byte_perm(u, 0x64646464u, 0x4140), y = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 a = __hsub2(*reinterpret_cast<__half2*>(&x), off), c = __hsub2(*reinterpret_cast<__half2*>(&y), off);
    lo = *reinterpret_cast<const uint32_t*>(&a);
    hi = *reinterpret_cast<const uint32_t*>(&c);
  }
}

// Four columns of the finished row i of KV head h; a row without keys, or one that does not exist, is zero.
__device__ __forceinline__ void kv8_store_row(const Kv8AttnArgs& a, int b, int h, int i, bool exists, float L, int c4, const float4& o) {
  const float inv = 1.f / L;
  const bool on = exists && L != 0.f;
  const __nv_bfloat162 x = __floats2bfloat162_rn(on ? o.x * inv : 0.f, on ? o.y * inv : 0.f);
  const __nv_bfloat162 y = __floats2bfloat162_rn(on ? o.z * inv : 0.f, on ? o.w * inv : 0.f);
  bf16* dst = a.out + ((size_t)((long long)b * a.rows + i / a.G) * a.hq + h * a.G + i % a.G) * a.c.dh + c4 * 4;
  DART_CHECK(i >= 0 && i < a.rows * a.G && b < a.batch && h < a.c.hkv && c4 * 4 < a.c.dh, a.status)
  *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
}

}  // namespace dart
