// Append to the paged 8-bit cache: new bf16 rows (a prompt, a token, the accepted path of a draft tree) are rounded to
// 8 bits with one power-of-two scale per (layer, page, KV head) and written into the pages.
//
// The scale is the smallest power of two that fits the block's largest finite value; e4m3 is a floating format, so a
// power of two costs it no precision, and for both formats it makes x / s exact: the one rounding is the one to 8 bits,
// and re-rounding a page's older codes when its scale grows is a shift of their exponents (e4m3: exact unless a code
// leaves the normal range).
#include "kv8.cuh"

namespace dart {

// Exponent of the smallest power of two s >= 2^-64 with value <= qmax * s; `bits`: the value's bf16 bits (finite, >= 0).
__device__ __forceinline__ int kv8_scale_exp(uint32_t bits, int format) {
  const int E = (int)(bits >> 7), M = (int)(bits & 127);
  const int k = format == KV8_E4M3 ? E - 135 + (M > 96) : E - 133 + (M > 126);   // 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
  return max(k, -64);
}

// Four values to four codes.  e4m3: round to nearest even, saturating; NaN stays NaN.  int8: the same, NaN becomes 0.
__device__ __forceinline__ uint32_t kv8_pack4(float x0, float x1, float x2, float x3, int format) {
  if (format == KV8_E4M3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x0, x1), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x2, x3), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
  }
  auto one = [](float x) { return (uint32_t)(min(max(__float2int_rn(x), -127), 127) & 255); };
  return one(x0) | (one(x1) << 8) | (one(x2) << 16) | (one(x3) << 24);
}
__device__ __forceinline__ float kv8_value(uint32_t code, int format) {
  return format == KV8_E4M3 ? __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3))) : (float)(int8_t)code;
}

constexpr int kApThreads = 256;
constexpr int kApPieces = 128 * 128 / 8 / kApThreads;   // 16-byte pieces of a page of one head that a thread holds

// One block per (layer, batch entry, touched page, KV head, K or V).
__global__ void __launch_bounds__(kApThreads) kv8_append_kernel(const __grid_constant__ Kv8AppendArgs a, long long units) {
  __shared__ uint32_t sh_max[kApThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    long long x = u;
    const int is_v = (int)(x & 1); x >>= 1;
    const int h = (int)(x % a.hkv); x /= a.hkv;
    const int w = (int)(x % a.windows); x /= a.windows;
    const int b = (int)(x % a.batch), layer = (int)(x / a.batch);
    const int slot = a.slots != nullptr ? a.slots[b] : b;
    const int n = a.n_append != nullptr ? a.n_append[b] : a.max_append;
    bool bad = slot < 0 || slot >= a.max_seqs || n < 0 || n > a.max_append;
    const int len = bad ? 0 : a.seq_lens[slot];
    if (len < 0 || (long long)len + n > (long long)a.max_pages * a.pt) bad = true;
    int twice = 0;
    if (a.slots != nullptr)
      for (int t = tid; t < b; t += kApThreads) twice |= a.slots[t] == slot;
    if (__syncthreads_or(twice)) bad = true;
    const int col = len / a.pt + w, first = col * a.pt;
    if (bad || n == 0 || first >= len + n) {
      if (bad && tid == 0) kv8_report(a.status, KV8_BAD_ARG);
      continue;
    }
    const int page = a.table[(size_t)slot * a.max_pages + col];
    if (page < 0 || page >= a.n_pages) {
      if (tid == 0) kv8_report(a.status, KV8_BAD_ARG);
      continue;
    }
    const int lo = max(len - first, 0), hi = min(a.pt, len + n - first);       // the new rows of this page
    const size_t ph = ((size_t)layer * a.n_pages + page) * a.hkv + h;
    uint8_t* codes = (is_v ? a.v : a.k) + ph * a.pt * a.dh;
    float* scale = (is_v ? a.vs : a.ks) + ph;
    const bf16* src = (is_v ? a.v_new : a.k_new) + (size_t)layer * a.layer_stride + (size_t)h * a.dh;
    const int cpr = a.dh / 8, pieces = (hi - lo) * cpr;
    uint4 v[kApPieces];
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < kApPieces; ++i) {
      const int e = tid + i * kApThreads;
      if (e < pieces) {
        const int j = first + lo + e / cpr - len;
        int row = a.row_index != nullptr ? a.row_index[(size_t)b * a.max_append + j] : j;
        if (row < 0 || row >= a.rows) { kv8_report(a.status, KV8_BAD_ARG); row = 0; }
        v[i] = *reinterpret_cast<const uint4*>(src + (size_t)((long long)b * a.rows + row) * a.row_stride + (e % cpr) * 8);
        const uint32_t wd[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t x0 = wd[q] & 0x7fffu, x1 = (wd[q] >> 16) & 0x7fffu;
          big = max(big, max(x0 < 0x7f80u ? x0 : 0u, x1 < 0x7f80u ? x1 : 0u));
        }
      }
    }
    const float was = first < len ? *scale : 0.f;
    big = __reduce_max_sync(0xffffffffu, big);
    if (lane == 0) sh_max[warp] = big;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kApThreads / 32; ++i) big = max(big, sh_max[i]);
    const int k = kv8_scale_exp(big, a.format);
    const float need = kv8_pow2(k), s = fmaxf(need, was);
    const bool exact = s == need || (__float_as_uint(s) & 0x7fffffu) == 0u;    // a power of two: the reciprocal is exact
    const float inv = 1.f / s;
#pragma unroll
    for (int i = 0; i < kApPieces; ++i) {
      const int e = tid + i * kApThreads;
      if (e < pieces) {
        const uint32_t wd[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
        float f[8];
#pragma unroll
        for (int q = 0; q < 4; ++q) { f[2 * q] = __uint_as_float(wd[q] << 16); f[2 * q + 1] = __uint_as_float(wd[q] & 0xffff0000u); }
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] = exact ? f[q] * inv : __fdiv_rn(f[q], s);
        *reinterpret_cast<uint2*>(codes + (size_t)lo * a.dh + (size_t)e * 8) =
            make_uint2(kv8_pack4(f[0], f[1], f[2], f[3], a.format), kv8_pack4(f[4], f[5], f[6], f[7], a.format));
      }
    }
    if (first < len && s != was) {     // the page's older codes, to the larger scale
      const float ratio = was / s;
      for (int e = tid; e < lo * a.dh / 4; e += kApThreads) {
        uint32_t* c = reinterpret_cast<uint32_t*>(codes) + e;
        const uint32_t o = *c;
        *c = kv8_pack4(kv8_value(o & 255, a.format) * ratio, kv8_value((o >> 8) & 255, a.format) * ratio,
                       kv8_value((o >> 16) & 255, a.format) * ratio, kv8_value(o >> 24, a.format) * ratio, a.format);
      }
    }
    if (tid == 0) *scale = s;
    __syncthreads();                   // sh_max is reused
  }
}

cudaError_t launch_kv8_append(const Kv8AppendArgs& a, cudaStream_t st) {
  const long long units = (long long)a.n_layers * a.batch * a.windows * a.hkv * 2;
  const unsigned grid = (unsigned)(units < (1ll << 30) ? units : (1ll << 30));
  kv8_append_kernel<<<grid, kApThreads, 0, st>>>(a, units);
  return cudaGetLastError();
}

}  // namespace dart
