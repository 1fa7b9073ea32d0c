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
template <int FMT>
__device__ __forceinline__ int kv8_scale_exp(uint32_t bits) {
  const int E = (int)(bits >> 7), M = (int)(bits & 127);
  const int k = FMT == KV8_E4M3 ? E - 135 + (M > 96) : E - 133 + (M > 126);   // 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
  return max(k, -64);
}

// Four values to four codes.  e4m3: round to nearest even, saturating; NaN stays NaN.  int8: the same (NaN becomes 0), for
// values of at least -127.5.
template <int FMT>
__device__ __forceinline__ uint32_t kv8_pack4(float x0, float x1, float x2, float x3) {
  if (FMT == KV8_E4M3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x0, x1), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x2, x3), __NV_SATFINITE, __NV_E4M3);
    return __byte_perm(lo, hi, 0x5410);
  }
  uint32_t d;
  asm("{\n.reg .b32 t;\ncvt.pack.sat.s8.s32.b32 t, %4, %3, 0;\ncvt.pack.sat.s8.s32.b32 %0, %2, %1, t;\n}"
      : "=r"(d) : "r"(__float2int_rn(x0)), "r"(__float2int_rn(x1)), "r"(__float2int_rn(x2)), "r"(__float2int_rn(x3)));
  return d;
}
template <int FMT>
__device__ __forceinline__ float kv8_value(uint32_t code) {
  return FMT == KV8_E4M3 ? __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3))) : (float)(int8_t)code;
}

// One team of threads per (layer, batch entry, touched page, KV head, K or V): a warp where a call adds at most 16 rows of
// 128 to a page (a decoding step, an accepted path), else a block of 128.  What bounds both is latency, not bytes: length
// -> rows and page id -> scale -> codes is a chain of three dependent reads of about a microsecond each, so the rows of
// a unit are all requested at once, before the page is known, and stay in registers between the maximum and the rounding,
// and the units in flight have to fill the GPU: four per block of warp teams, and no more registers than the page size
// asks for in a block team (PIECES 16-byte pieces per thread).  Next to the latencies it is instructions: a page's
// largest value comes from 16-bit three-way maxima of the raw words, rows are found by adding a stride.
// Measured (device time, back to back in a CUDA graph; through Python 8.2 and 14.5): 16 accepted paths x 16 layers x 8 heads (8.3 MB)
// 7.2 us, 39 with a block of 256 per unit; 4 x 2047 prompt rows x 8 heads (50 MB) 13.75 us = 0.56 of the copy peak, 35 with the rows read after the page, 20 with element-wise maxima, 14.9
// in blocks of 256, 19 in warp teams; strips of pages per block, the next page's rows in flight: 32.
constexpr int kApThreads = 128;

template <int TEAM>
__device__ __forceinline__ void team_sync() {
  if (TEAM == 32) __syncwarp(); else __syncthreads();
}
template <int TEAM>
__device__ __forceinline__ bool team_any(bool x) {
  return TEAM == 32 ? __any_sync(0xffffffffu, x) : __syncthreads_or(x);
}

template <int FMT, int DH, int TEAM, int PIECES>
__global__ void __launch_bounds__(kApThreads) kv8_append_kernel(const __grid_constant__ Kv8AppendArgs a) {
  __shared__ uint32_t sh_max[kApThreads / 32];
  constexpr int kPer = DH / 8;                     // pieces of a row
  const int tid = threadIdx.x % TEAM, lane = threadIdx.x & 31;
  const int b = blockIdx.y, layer = blockIdx.z, heads2 = 2 * a.hkv;
  const int unit = blockIdx.x * (kApThreads / TEAM) + threadIdx.x / TEAM;
  const int w = unit / heads2, is_v = (unit % heads2) / a.hkv, h = unit % a.hkv;      // neighbours: the heads of a row
  if (w >= a.windows) return;                       // (whole teams)
  const int slot = a.slots != nullptr ? a.slots[b] : b;
  const int n = a.n_append != nullptr ? a.n_append[b] : a.max_append;
  bool bad = slot < 0 || slot >= a.max_seqs || n < 0 || n > a.max_append;
  const int len = bad ? 0 : a.seq_lens[slot];
  if (len < 0 || (long long)len + n > (long long)a.max_pages * a.pt) bad = true;
  if (n == 0 && !bad) return;                      // (and claims no slot: the padding of a batch)
  if (a.slots != nullptr) {                        // a slot that an entry with rows named before is skipped
    bool twice = false;
    for (int t = tid; t < b; t += TEAM) twice |= a.slots[t] == slot && (a.n_append == nullptr || a.n_append[t] != 0);
    if (team_any<TEAM>(twice)) bad = true;
  }
  if (bad) {
    if (tid == 0) kv8_report(a.status, KV8_BAD_ARG);
    return;
  }
  const bf16* src = (is_v ? a.v_new : a.k_new) + (size_t)layer * a.layer_stride + (size_t)h * DH;
  // the page of column `col` and the rows that go there
  struct Unit { int page, lo, pieces; uint4 v[PIECES]; };
  auto request = [&](int col, Unit& x) {
    const int first = col * a.pt;
    x.lo = max(len - first, 0);
    x.pieces = max(min(a.pt, len + n - first) - x.lo, 0) * kPer;
    if (x.pieces == 0) return;
    x.page = a.table[(size_t)slot * a.max_pages + col];
    const int j0 = first + x.lo + tid / kPer - len;      // this thread's first row; the next are TEAM / kPer rows apart
    const bf16* p = src + (size_t)((long long)b * a.rows + j0) * a.row_stride + (tid % kPer) * 8;
    const size_t step = (size_t)(TEAM / kPer) * a.row_stride;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      if (tid + i * TEAM < x.pieces) {
        const bf16* from = p + i * step;
        if (a.row_index != nullptr) {
          int row = a.row_index[(size_t)b * a.max_append + j0 + i * (TEAM / kPer)];
          if (row < 0 || row >= a.rows) { kv8_report(a.status, KV8_BAD_ARG); row = 0; }
          from = src + (size_t)((long long)b * a.rows + row) * a.row_stride + (tid % kPer) * 8;
        }
        x.v[i] = __ldg(reinterpret_cast<const uint4*>(from));
      }
    }
  };
  auto store = [&](int col, const Unit& x) {
    if (x.page < 0 || x.page >= a.n_pages) {
      if (tid == 0) kv8_report_first(a.status, KV8_BAD_ARG);
      return;
    }
    const size_t ph = ((size_t)layer * a.n_pages + x.page) * a.hkv + h;
    uint8_t* codes = (is_v ? a.v : a.k) + ph * a.pt * DH;
    float* scale = (is_v ? a.vs : a.ks) + ph;
    const bool held = col * a.pt < len;            // the page already holds rows of the sequence
    const int names = a.ref != nullptr ? a.ref[x.page] : 1;
    const float was = held ? *scale : 0.f;
    if (names != 1) {                              // other sequences read this page (or nobody holds it)
      if (tid == 0) kv8_report_first(a.status, KV8_BAD_ARG);
      return;
    }
    // the largest |x|: bits of both halves of all words, a three-way 16-bit maximum per two words
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      if (tid + i * TEAM < x.pieces) {
        top = __vimax3_u16x2(top, x.v[i].x & 0x7fff7fffu, x.v[i].y & 0x7fff7fffu);
        top = __vimax3_u16x2(top, x.v[i].z & 0x7fff7fffu, x.v[i].w & 0x7fff7fffu);
      }
    uint32_t big = max(top & 0xffffu, top >> 16);
    const bool odd = big >= 0x7f80u;               // something is not finite: the largest of the rest, element by element
    if (odd) {
      big = 0;
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        if (tid + i * TEAM < x.pieces) big = kv8_max_finite(big, x.v[i]);
    }
    big = __reduce_max_sync(0xffffffffu, big);
    if (TEAM > 32) {
      if (lane == 0) sh_max[threadIdx.x >> 5] = big;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < TEAM / 32; ++i) big = max(big, sh_max[i]);
    }
    team_sync<TEAM>();                             // everybody has read the old scale
    const float need = kv8_pow2(kv8_scale_exp<FMT>(big)), s = fmaxf(need, was);
    const bool exact = (__float_as_uint(s) & 0x7fffffu) == 0u;               // a power of two: the reciprocal is exact
    const float inv = 1.f / s;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = tid + i * TEAM;
      if (e < x.pieces) {
        const uint32_t wd[4] = {x.v[i].x, x.v[i].y, x.v[i].z, x.v[i].w};
        float f[8];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f[2 * q] = __uint_as_float(wd[q] << 16) * inv;
          f[2 * q + 1] = __uint_as_float(wd[q] & 0xffff0000u) * inv;
        }
        if (!exact || odd) {                       // a scale that is no power of two, or infinities
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            f[q] = __uint_as_float(q & 1 ? wd[q / 2] & 0xffff0000u : wd[q / 2] << 16);
            f[q] = __fdiv_rn(f[q], s);
            if (FMT == KV8_INT8 && f[q] < -127.f) f[q] = -127.f;
          }
        }
        DART_CHECK(x.lo >= 0 && x.lo * kPer + e < a.pt * kPer && layer < a.n_layers && h < a.hkv, a.status)
        *reinterpret_cast<uint2*>(codes + (size_t)x.lo * DH + (size_t)e * 8) =
            make_uint2(kv8_pack4<FMT>(f[0], f[1], f[2], f[3]), kv8_pack4<FMT>(f[4], f[5], f[6], f[7]));
      }
    }
    if (held && s != was) {          // the page's older codes, to the larger scale
      const float ratio = was / s;
      for (int e = tid; e < x.lo * DH / 4; e += TEAM) {
        uint32_t* c = reinterpret_cast<uint32_t*>(codes) + e;
        const uint32_t o = *c;
        DART_CHECK(e * 4 < a.pt * DH, a.status)
        *c = kv8_pack4<FMT>(kv8_value<FMT>(o & 255) * ratio, kv8_value<FMT>((o >> 8) & 255) * ratio, kv8_value<FMT>((o >> 16) & 255) * ratio,
                            kv8_value<FMT>(o >> 24) * ratio);
      }
    }
    if (tid == 0 && s != was) *scale = s;
  };
  const int col0 = len / a.pt, end = (len + n - 1) / a.pt + 1;      // columns that get rows
  Unit x;
  const int col = col0 + w;
  if (col >= end) return;
  request(col, x);
  store(col, x);
}

namespace {
template <int FMT, int DH, int TEAM, int PIECES>
cudaError_t launch(const Kv8AppendArgs& a, cudaStream_t st) {
  const long long units = (long long)a.windows * 2 * a.hkv, teams = kApThreads / TEAM;
  kv8_append_kernel<FMT, DH, TEAM, PIECES><<<dim3((unsigned)((units + teams - 1) / teams), a.batch, a.n_layers), kApThreads, 0, st>>>(a);
  return cudaGetLastError();
}
template <int FMT, int DH>
cudaError_t launch_rows(const Kv8AppendArgs& a, cudaStream_t st) {
  const int pieces = (a.max_append < a.pt ? a.max_append : a.pt) * (DH / 8);      // of the fullest page
  if (pieces <= 32) return launch<FMT, DH, 32, 1>(a, st);
  if (pieces <= 256) return launch<FMT, DH, 32, 8>(a, st);
  if (pieces <= 512) return launch<FMT, DH, 128, 4>(a, st);
  if (pieces <= 1024) return launch<FMT, DH, 128, 8>(a, st);
  return launch<FMT, DH, 128, 16>(a, st);
}
}  // namespace

cudaError_t launch_kv8_append(const Kv8AppendArgs& a, cudaStream_t st) {
  if (a.format == KV8_E4M3) return a.dh == 128 ? launch_rows<KV8_E4M3, 128>(a, st) : launch_rows<KV8_E4M3, 64>(a, st);
  return a.dh == 128 ? launch_rows<KV8_INT8, 128>(a, st) : launch_rows<KV8_INT8, 64>(a, st);
}

}  // namespace dart
