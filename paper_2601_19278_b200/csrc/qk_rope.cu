// Norms of queries and keys for each head with the position rotation in the same pass (include/dart.h: dart_qk_norm_rope).
//
//   y = x * rsqrt(mean(x^2) + eps) * w,      (y_a, y_b) -> (y_a cos - y_b sin, y_a sin + y_b cos),   angle_i = position * f_i
//
// per head, in fp32, with one rounding at the end; pairs (a, b) are (i, i + n/2) or neighbours (2i, 2i + 1) of the first n
// elements, the rest of the head is not rotated.  Angles run to 10^5 and more radians, where an fp32 product has lost them
// (2^-24 of 131072 is 0.008): frequencies are turns per position as 64-bit fractions, so that position * f wraps by itself and
// has the angle to 2^-32 of a turn (dart_rope_frequencies); as an fp32 number of half turns it is off by up to 2^-26 of a turn, at any position.
//
// What bounds it is the bytes, each read and written once.  A head is 16 elements to a lane (two 8-element chunks that are each
// other's partners, so that a pair never crosses lanes): 128-byte segments, four or eight heads to a warp, and a sum over
// d / 16 lanes.  A block takes one token; its d / 2 sines are computed once for all heads, behind the loads of the heads.
// 8191 rows of 48 bf16 heads of 128 out of a QKV matrix: 34.8 us = 5.8 TB/s, 0.88 of the copy peak (a plain copy of as much 33.2); one
// operation to an instruction 37.5; more or fewer registers (6 to 8 blocks to an SM), 64 threads to a block and streaming stores change nothing,
// 256 threads take 50.
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include "../../include/dart.h"
#include "common.cuh"
#include "kernels.h"

namespace dart {

struct QkRopeArgs {
  int batch, rows, hq, hk, rotary, max_seqs;
  long long q_stride, k_stride, qo_stride, ko_stride;      // elements from row to row
  const void *q, *k;
  void *q_out, *k_out;
  const void *q_norm, *k_norm;                             // null: no norm
  float eps;
  const unsigned long long* freqs;
  const int *positions, *seq_lens, *slots, *n_rows;
  int* status;
};

constexpr int kRopeThreads = 128;

// Eight elements as four pairs of floats, and back.  (Arithmetic goes by pairs, two operations to an instruction.)
template <class T>
struct Chunk8;
template <>
struct Chunk8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
  __device__ __forceinline__ void get(float2 (&f)[4]) const {
    f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w); f[2] = make_float2(b.x, b.y); f[3] = make_float2(b.z, b.w);
  }
  static __device__ __forceinline__ void store(float* p, const float2 (&f)[4]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
  }
};
template <>
struct Chunk8<bf16> {
  uint4 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float2 (&f)[4]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  static __device__ __forceinline__ void store(bf16* p, const float2 (&f)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __float22bfloat162_rn(f[i]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Chunk8<__half> {
  uint4 v;
  __device__ __forceinline__ void load(const __half* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float2 (&f)[4]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    }
  }
  static __device__ __forceinline__ void store(__half* p, const float2 (&f)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __float22half2_rn(f[i]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// NH heads to a thread, all of them requested before anything else; blockIdx.y takes the next NH * (heads of a block) heads.
// PART: heads that are rotated in part.  Lanes behind the rotated elements leave theirs alone; turned by an angle of 0, an infinity or NaN would
// spread to the element beside it.  (The same branch in front of heads that are rotated whole: the prompt below 34.8 -> 35.8 us; a select instead of it 38.7.)
template <class T, int DH, int NH, bool PART>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_kernel(const __grid_constant__ QkRopeArgs a, int interleaved) {
  constexpr int kLanes = DH / 16, kHeads = kRopeThreads / kLanes;      // lanes of a head, heads that a block has at a time
  __shared__ __align__(16) float s_cos[DH / 2], s_sin[DH / 2];
  const int tid = threadIdx.x, l = tid % kLanes, token = blockIdx.x;
  const int b = token / a.rows, r = token - b * a.rows;
  pdl_wait();
  pdl_trigger();
  const int nr = a.n_rows != nullptr ? a.n_rows[b] : a.rows;
  int pos;
  bool bad = nr < 0 || nr > a.rows;
  if (a.positions != nullptr) {
    pos = a.positions[token];
  } else {
    const int slot = a.slots != nullptr ? a.slots[b] : b;
    if (slot < 0 || slot >= a.max_seqs) bad = true;
    const int len = bad ? 0 : a.seq_lens[slot];
    if (len < 0 || len > 0x7fffffff - r) bad = true;
    pos = bad ? -1 : len + r;
  }
  if (bad) {
    if (tid == 0 && blockIdx.y == 0 && a.status != nullptr) atomicExch(a.status, (int)DART_ERR_INVALID_ARG);
    return;
  }
  if (r >= nr || pos < 0) return;

  // chunk numbers of this lane: partners, or two that pass
  const int n8 = a.rotary / 8, pairs = n8 / 2;                           // rotated chunks
  const bool turns = !PART || l < pairs;
  const int c0 = turns ? (interleaved ? 2 * l : l) : n8 + 2 * (l - pairs), c1 = turns && !interleaved ? l + pairs : c0 + 1;
  Chunk8<T> x0[NH], x1[NH];
  const int first = blockIdx.y * (NH * kHeads) + tid / kLanes;
#pragma unroll
  for (int i = 0; i < NH; ++i) {
    const int h = first + i * kHeads;
    if (h >= a.hq + a.hk) { x0[i] = x1[i] = Chunk8<T>{}; continue; }
    const T* src = h < a.hq ? static_cast<const T*>(a.q) + (size_t)token * a.q_stride + (size_t)h * DH
                            : static_cast<const T*>(a.k) + (size_t)token * a.k_stride + (size_t)(h - a.hq) * DH;
    x0[i].load(src + c0 * 8);
    x1[i].load(src + c1 * 8);
  }
  for (int i = tid; i < a.rotary / 2; i += kRopeThreads) {
    const int turn = (int)((a.freqs[i] * (unsigned long long)pos) >> 32);      // 2^-32 turns = 2^-31 pi
    sincospif((float)turn * 4.656612873077393e-10f, &s_sin[i], &s_cos[i]);
  }
  __syncthreads();
  float2 cs[4], sn[4], ns[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    cs[e] = turns ? *reinterpret_cast<const float2*>(&s_cos[8 * l + 2 * e]) : make_float2(1.f, 1.f);
    sn[e] = turns ? *reinterpret_cast<const float2*>(&s_sin[8 * l + 2 * e]) : make_float2(0.f, 0.f);
    ns[e] = make_float2(-sn[e].x, -sn[e].y);
  }
#pragma unroll
  for (int i = 0; i < NH; ++i) {
    const int h = first + i * kHeads;
    const bool on = h < a.hq + a.hk, is_q = h < a.hq;
    float2 f0[4], f1[4];
    x0[i].get(f0);                         // (of a head that does not exist: whatever, and nothing is stored)
    x1[i].get(f1);
    if (a.q_norm != nullptr) {             // (both norms or neither)
      float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int e = 0; e < 4; ++e) s2 = __ffma2_rn(f0[e], f0[e], __ffma2_rn(f1[e], f1[e], s2));
      float ss = s2.x + s2.y;
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float inv = rsqrtf(ss * (1.f / DH) + a.eps);
      if (on) {
        const T* norm = static_cast<const T*>(is_q ? a.q_norm : a.k_norm);
        const float2 inv2 = make_float2(inv, inv);
        Chunk8<T> w;
        float2 g[4];
        w.load(norm + c0 * 8);
        w.get(g);
#pragma unroll
        for (int e = 0; e < 4; ++e) f0[e] = __fmul2_rn(f0[e], __fmul2_rn(inv2, g[e]));
        w.load(norm + c1 * 8);
        w.get(g);
#pragma unroll
        for (int e = 0; e < 4; ++e) f1[e] = __fmul2_rn(f1[e], __fmul2_rn(inv2, g[e]));
      }
    }
    if (!on) continue;
    float2 y0[4], y1[4];
    if (!turns) {
#pragma unroll
      for (int e = 0; e < 4; ++e) { y0[e] = f0[e]; y1[e] = f1[e]; }
    } else if (interleaved) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {        // pair 4 x + e of this lane's eight
        const float c = e & 1 ? cs[e / 2].y : cs[e / 2].x, n = e & 1 ? sn[e / 2].y : sn[e / 2].x;
        y0[e] = make_float2(f0[e].x * c - f0[e].y * n, f0[e].x * n + f0[e].y * c);
        const float d = e & 1 ? cs[2 + e / 2].y : cs[2 + e / 2].x, m = e & 1 ? sn[2 + e / 2].y : sn[2 + e / 2].x;
        y1[e] = make_float2(f1[e].x * d - f1[e].y * m, f1[e].x * m + f1[e].y * d);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y0[e] = __ffma2_rn(f0[e], cs[e], __fmul2_rn(f1[e], ns[e]));
        y1[e] = __ffma2_rn(f0[e], sn[e], __fmul2_rn(f1[e], cs[e]));
      }
    }
    T* dst = is_q ? static_cast<T*>(a.q_out) + (size_t)token * a.qo_stride + (size_t)h * DH
                  : static_cast<T*>(a.k_out) + (size_t)token * a.ko_stride + (size_t)(h - a.hq) * DH;
    DART_CHECK(token < a.batch * a.rows && c0 * 8 < DH && c1 * 8 < DH, a.status) {
      Chunk8<T>::store(dst + c0 * 8, y0);
      Chunk8<T>::store(dst + c1 * 8, y1);
    }
  }
}

namespace {

template <class T, int DH, bool PART>
cudaError_t launch(const QkRopeArgs& a, int interleaved, cudaStream_t st) {
  constexpr int kHeads = kRopeThreads / (DH / 16);
  const int tokens = a.batch * a.rows, passes = (a.hq + a.hk + kHeads - 1) / kHeads;
  // Heads of a thread: as many as there are up to four, so that a token's angles are computed once; one where the tokens alone
  // leave SMs idle and a call is a chain of latencies.
  const int groups = (passes + 3) / 4, nh = tokens * passes <= 148 ? 1 : (passes + groups - 1) / groups;
  const dim3 grid(tokens, (passes + nh - 1) / nh);
  switch (nh) {
    case 1: return launch_ahead(qk_norm_rope_kernel<T, DH, 1, PART>, grid, kRopeThreads, 0, st, a, interleaved);
    case 2: return launch_ahead(qk_norm_rope_kernel<T, DH, 2, PART>, grid, kRopeThreads, 0, st, a, interleaved);
    case 3: return launch_ahead(qk_norm_rope_kernel<T, DH, 3, PART>, grid, kRopeThreads, 0, st, a, interleaved);
    default: return launch_ahead(qk_norm_rope_kernel<T, DH, 4, PART>, grid, kRopeThreads, 0, st, a, interleaved);
  }
}

template <class T>
cudaError_t launch_dim(const QkRopeArgs& a, int dim, int interleaved, cudaStream_t st) {
  if (a.rotary < dim) return dim == 128 ? launch<T, 128, true>(a, interleaved, st) : launch<T, 64, true>(a, interleaved, st);
  return dim == 128 ? launch<T, 128, false>(a, interleaved, st) : launch<T, 64, false>(a, interleaved, st);
}

bool aligned(const void* p, unsigned n) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool null_or_aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace
}  // namespace dart

using namespace dart;

extern "C" int dart_rope_frequencies(const double* inv_freq, int32_t n, uint64_t* out) {
  if (inv_freq == nullptr || out == nullptr || n < 1 || n > 64) return DART_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i)
    if (!(fabs(inv_freq[i]) <= 3.141592653589793)) return DART_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    // turns per position as a fraction of 2^64 (x86's 64-bit significand: off by at most 2^-64 of it), negative ones wrapped
    const long double turns = (long double)fabs(inv_freq[i]) / 6.283185307179586476925286766559L;
    const uint64_t f = (uint64_t)(turns * 18446744073709551616.0L + 0.5L);
    out[i] = inv_freq[i] < 0.0 ? 0 - f : f;
  }
  return DART_OK;
}

extern "C" int dart_qk_norm_rope(const dart_qk_rope_in* in, void* cuda_stream) {
  if (in == nullptr || in->batch < 1 || in->rows < 1 || (long long)in->batch * in->rows > (1 << 24) || in->n_q_heads < 1 || in->n_q_heads > 1024 ||
      in->n_k_heads < 0 || in->n_k_heads > 1024 || (in->head_dim != 64 && in->head_dim != 128) || in->rotary_dim < 16 ||
      in->rotary_dim > in->head_dim || in->rotary_dim % 16 != 0 || (in->interleaved != 0 && in->interleaved != 1))
    return DART_ERR_INVALID_ARG;
  if (in->dtype != DART_BF16 && in->dtype != DART_FP16 && in->dtype != DART_FP32) return DART_ERR_INVALID_ARG;
  const int unit = in->dtype == DART_FP32 ? 4 : 8;                       // elements of 16 bytes
  const int64_t wq = (int64_t)in->n_q_heads * in->head_dim, wk = (int64_t)in->n_k_heads * in->head_dim;
  if (!aligned(in->q, 16) || !aligned(in->q_out, 16) || in->q_stride < wq || in->q_stride % unit != 0 || in->q_out_stride < wq ||
      in->q_out_stride % unit != 0)
    return DART_ERR_INVALID_ARG;
  if (in->n_k_heads > 0 && (!aligned(in->k, 16) || !aligned(in->k_out, 16) || in->k_stride < wk || in->k_stride % unit != 0 ||
                            in->k_out_stride < wk || in->k_out_stride % unit != 0))
    return DART_ERR_INVALID_ARG;
  if (!null_or_aligned(in->q_norm, 16) || !null_or_aligned(in->k_norm, 16) ||
      (in->n_k_heads > 0 && (in->q_norm == nullptr) != (in->k_norm == nullptr)) || !(in->eps >= 0.f) || !aligned(in->freqs, 8))
    return DART_ERR_INVALID_ARG;
  if (in->positions != nullptr ? in->seq_lens != nullptr || in->slots != nullptr
                               : in->seq_lens == nullptr || in->max_seqs < 1 || (in->slots == nullptr && in->batch > in->max_seqs))
    return DART_ERR_INVALID_ARG;
  if (!null_or_aligned(in->positions, 4) || !null_or_aligned(in->seq_lens, 4) || !null_or_aligned(in->slots, 4) || !null_or_aligned(in->n_rows, 4) ||
      !null_or_aligned(in->status, 4))
    return DART_ERR_INVALID_ARG;
  const int arch = check_sm100();
  if (arch != DART_OK) return arch;
  QkRopeArgs a;
  memset(&a, 0, sizeof(a));
  a.batch = in->batch; a.rows = in->rows; a.hq = in->n_q_heads; a.hk = in->n_k_heads; a.rotary = in->rotary_dim; a.max_seqs = in->max_seqs;
  a.q_stride = in->q_stride; a.k_stride = in->k_stride; a.qo_stride = in->q_out_stride; a.ko_stride = in->k_out_stride;
  a.q = in->q; a.k = in->k; a.q_out = in->q_out; a.k_out = in->k_out;
  a.q_norm = in->q_norm; a.k_norm = in->k_norm; a.eps = in->eps;
  a.freqs = reinterpret_cast<const unsigned long long*>(in->freqs);
  a.positions = in->positions; a.seq_lens = in->seq_lens; a.slots = in->slots; a.n_rows = in->n_rows; a.status = in->status;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = in->dtype == DART_BF16 ? launch_dim<bf16>(a, in->head_dim, in->interleaved, st)
                        : in->dtype == DART_FP16 ? launch_dim<__half>(a, in->head_dim, in->interleaved, st)
                                                 : launch_dim<float>(a, in->head_dim, in->interleaved, st);
  if (e == cudaSuccess) return DART_OK;
  record_global_cuda_error(e);
  return DART_ERR_CUDA;
}
