// Attention over the paged 8-bit cache (include/dart.h: dart_kv8_attention): planning, the kernel for few rows, the join.
//
//   out[r] = sum_y softmax_y(q[r] . k[y] / sqrt(d)) v[y],   k[y] = s_k * code,  v[y] = s_v * code
//
// Codes of both formats are exact in fp16, and so is a bf16 query or new row once divided by a power of two near its
// largest element, but for elements below 2^-17 of that (off by up to 2^-25 of it; new values 2^-23 and 2^-31, or less): both
// products run on fp16 tensor-core instructions with next to nothing rounded but the weights.  The scales
// never touch the codes: with c = log2(e) / sqrt(d) times the query's power of two, a key of a page with scales s_k, s_v
// enters as
//   x = (c s_k) (q . code) + log2(s_v),     P = 2^(x - m + 9),     2^9 l += P / s_v,     O += P code,     out = O / (2^9 l)
// where m follows the largest x (not the largest score): P is the key's weight times its value's scale, 2^15 at most, so its
// rounding to fp16 is 2^-11 of what the key contributes, however far apart the pages' scales are, or, for P below 2^-14, 2^-34 of
// the largest weight times scale (kv8.cuh: kKv8Bias); over n keys that is at most n 2^-34 of the largest |v| on the
// scale of the heaviest key's page.  m, l and O are fp32.  New rows are keys with a power-of-two scale of their own
// (kv8.cuh: kv8_row_exp, kv8_lift).
//
// Rows of all query heads that share a KV head are one matrix (row r, head g of the group -> r * G + g).  Up to 24 such
// rows (32 with d = 64: kv8_stream_rows) run on kv8_attn_stream_kernel below: a stream of the cache at memory speed.  More rows run on tcgen05
// (kv8_attn_umma.cu).  A long key axis is split over CTAs; their partial (m, l, O) go through the workspace and
// kv8_combine_kernel joins them.
#include <string.h>

#include "kv8.cuh"

namespace dart {

// ---- few rows ---------------------------------------------------------------------------------------------------------
// What bounds it is the stream of K and V bytes, and that takes bytes in flight: about 60 KB per SM, which registers cannot
// hold beside the accumulators (with one group of 16 keys ahead in registers, 48 KB per SM, 64 ragged sequences took 126 us;
// from the rings 96 us = 5.9 TB/s, 0.91 of the copy peak).  Every warp therefore has a ring of its own in shared
// memory, kStStages groups of 16 keys deep, filled by 16-byte asynchronous copies; rows are laid out so that the reads below
// meet no bank twice.  From there every lane reads exactly the bytes that its own tensor-core fragments need:
//   S^T = K Q^T    mma m16n8k16 with the 16 keys as M.  The order of the contraction index is free as long as Q and K agree:
//                  lane t of a key's quad takes d = [t * DH/4, (t+1) * DH/4), whole 16-byte words of the key's row.
//   O^T = V^T P^T  the same instruction with d as M: its A operand wants pairs of neighbouring keys, which two bytes of
//                  two keys' words give by one byte permutation before the conversion; P^T is the first product's result
//                  transposed in 8 x 8 blocks (movmatrix).  Both products give a lane the same two rows, so m and l are its own.
// m moves only when a score exceeds it by 2^6: the common case has no shuffles at all.  Instructions count next to the bytes
// (with rows as M in the first product, half of M empty, and scales and addresses from global memory a group of 4 KB took 319
// of them and the batch of 64 tokens 120 us): scales, their logarithms and the page ids of the CTA's groups are laid out in
// shared memory once.
constexpr int kStWarps = 4, kStStages = 4;

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Place of the 16-byte chunk c of row r in a [16][DH] byte tile: lines of 128 bytes, chunks exchanged within a line so that
// lanes (g, t) that read chunk f(t) of rows g, or chunk g of rows 2t, meet different banks.
template <int DH>
__device__ __forceinline__ uint32_t st_place(int r, int c) {
  if (DH == 128) return r * 128 + ((c ^ (r & 7)) << 4);
  const int line = r >> 1;
  return line * 128 + (((((r & 1) << 2) | c) ^ ((line * 2) & 7)) << 4);
}

// Shared memory: the warps' rings, later their O; then the groups' scales and pages.
template <int DH, int NT>
constexpr __host__ __device__ int st_body() {
  return kStWarps * kStStages * 2 * 16 * DH > kStWarps * 8 * NT * DH * 4 ? kStWarps * kStStages * 2 * 16 * DH : kStWarps * 8 * NT * DH * 4;
}

// NT tiles of 8 rows.  With more of them the instructions per byte grow and registers run out (O and Q take 48 NT a thread at
// d = 128, 24 NT at 64), which sets how many CTAs fit an SM; tcgen05 converts a step's codes at one cost for 1 to 128 rows.
// Both sides, 8 KV heads, e4m3, us here and there: 16 sequences of 8192 keys, d = 128: 4 rows x 5 heads 88, 109; 32 rows 148
// (spilled), 110; d = 64: 6 x 4 61, 93; 8 x 4 72.5, 94.  64 of 2048, d = 128: 4 x 5 101, 148; d = 64: 8 x 4 86.5, 123.  New rows are
// the last warp's own, 16 at a time: 20 rows of one head 93, 110.  A single sequence of 8192 loses: d = 128, 4 x 5 18.7, 17.6, 20
// of one head 22.6, 17.7; d = 64, 8 x 4 16.4, 15.4.
// d = 64, 64 sequences of 2048 keys: four CTAs to an SM instead of three for 8 rows 37 us, 41; three instead of two for 16 rows
// 50, 57.
constexpr __host__ __device__ int kv8_stream_ctas(int dh, int nt) { return nt == 1 ? (dh == 64 ? 4 : 3) : nt == 2 && dh == 64 ? 3 : 2; }
constexpr __host__ __device__ int kv8_stream_rows(int dh) { return dh == 64 ? 32 : 24; }
template <int FMT, int DH, int NT>
__global__ void __launch_bounds__(kStWarps * 32, kv8_stream_ctas(DH, NT)) kv8_attn_stream_kernel(const __grid_constant__ Kv8AttnArgs a,
                                                                                        const Kv8Plan plan) {
  constexpr int MT = DH / 16, KW = DH / 16;     // d tiles of the second product; words of a lane's piece of a key
  constexpr int NR = 8 * NT;
  extern __shared__ __align__(16) unsigned char st_smem[];
  constexpr int kTile = 16 * DH;                                 // codes of 16 keys
  unsigned char* ring = st_smem + (threadIdx.x >> 5) * (kStStages * 2 * kTile);                       // this warp's
  float(*s_o)[NR][DH] = reinterpret_cast<float(*)[NR][DH]>(st_smem);                                  // in the end, all warps' O
  float4* s_group = reinterpret_cast<float4*>(st_smem + st_body<DH, NT>());     // per group of 16 keys: k's scale, log2 and (unbiased) reciprocal of v's, page id
  __shared__ float s_m[kStWarps][NR], s_l[kStWarps][NR];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int h = blockIdx.x, b = blockIdx.y, chunk_id = blockIdx.z;
  const Kv8Seq s = kv8_seq(a, b, threadIdx.x == 0 && h == 0 && chunk_id == 0);
  const int N = a.rows * a.G, Nv = s.rows * a.G;                  // rows of the call, rows that exist
  const Kv8Split sp = kv8_split_keys(s.len, plan.chunk);
  pdl_trigger();                                  // the join may be scheduled as SMs drain; it waits for this grid
  if (chunk_id >= sp.n) return;
  const int k0 = chunk_id * sp.per, k1 = min(s.len, k0 + sp.per), n_groups = (k1 - k0 + 15) / 16;
  const bool last = chunk_id == sp.n - 1;
  const size_t page_bytes = (size_t)a.c.hkv * a.c.pt * DH;
  const long long v_off = a.c.v - a.c.k;
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);
  // the copies of a group: 512 bytes of K or of V per instruction
  uint32_t put[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) put[i] = st_place<DH>((lane + 32 * i) / (DH / 16), (lane + 32 * i) % (DH / 16));
  auto request = [&](int gi, int stage, int page) {
    if (gi < n_groups) {
      const uint8_t* src = a.c.k + (size_t)page * page_bytes + (h * a.c.pt + ((k0 + 16 * gi) & (a.c.pt - 1))) * DH + lane * 16;
      const uint32_t dst = ring_s + stage * (2 * kTile);
#pragma unroll
      for (int i = 0; i < DH / 32; ++i) cp_async_16(dst + put[i], src + i * 512);
#pragma unroll
      for (int i = 0; i < DH / 32; ++i) cp_async_16(dst + kTile + put[i], src + v_off + i * 512);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // the first copies start as soon as their page ids are known, before everything else
#pragma unroll
  for (int i = 0; i < kStStages - 1; ++i) {
    const int gi = warp + i * kStWarps;
    request(gi, i, gi < n_groups ? kv8_page(a, s.slot, (k0 + 16 * gi) >> a.c.pt_log2) : 0);
  }
  for (int i = threadIdx.x; i < n_groups; i += kStWarps * 32) {
    const int page = kv8_page(a, s.slot, (k0 + 16 * i) >> a.c.pt_log2);
    const float sv = fmaxf(a.c.vs[(size_t)page * a.c.hkv + h], kv8_pow2(-100));
    s_group[i] = make_float4(a.c.ks[(size_t)page * a.c.hkv + h], __log2f(sv), kKv8Unbias / sv, __int_as_float(page));
  }

  // Q as the B operand: row g of each tile, d of this lane in the order of the K words; a power of two brings a row's
  // largest finite element to [1, 2)
  uint32_t q[NT][KW][2];
  float crow[NT][2];                              // of rows 2t, 2t + 1
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int i = g + 8 * n;
    const bool on = i < Nv;
    const int r = on ? i / a.G : 0;
    const bf16* qp = a.q + (size_t)((long long)b * a.rows + r) * a.q_stride + (size_t)(h * a.G + (on ? i - r * a.G : 0)) * DH + t * (DH / 4);
    uint4 raw[DH / 32];
    uint32_t big = 0;
#pragma unroll
    for (int e = 0; e < DH / 32; ++e) raw[e] = on ? *(reinterpret_cast<const uint4*>(qp) + e) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int e = 0; e < DH / 32; ++e) big = kv8_max_finite(big, raw[e]);
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
    const int ex = kv8_row_exp(big);
    const float c = a.scale_log2e * kv8_pow2(ex), inv = kv8_pow2(-ex);
    crow[n][0] = __shfl_sync(0xffffffffu, c, 8 * t);
    crow[n][1] = __shfl_sync(0xffffffffu, c, 8 * t + 4);
#pragma unroll
    for (int e = 0; e < DH / 32; ++e) {
      uint32_t f[4];
      kv8_bf16x8_to_half(raw[e], inv, f);
#pragma unroll
      for (int w = 0; w < 2; ++w) { q[n][2 * e + w][0] = f[2 * w]; q[n][2 * e + w][1] = f[2 * w + 1]; }   // word 2e + w: d 4 (2e + w) .. + 3
    }
  }
  __syncthreads();

  float o[MT][NT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) o[m][n][0] = o[m][n][1] = o[m][n][2] = o[m][n][3] = 0.f;
  float m_ref[NT][2], l[NT][2];                   // of rows 2t, 2t + 1
#pragma unroll
  for (int n = 0; n < NT; ++n) { m_ref[n][0] = m_ref[n][1] = -INFINITY; l[n][0] = l[n][1] = 0.f; }

  // x[n][4]: (key g, rows 2t, 2t+1), (key g + 8, the same rows), scaled, -inf where hidden.  Turns them into P (with its
  // bias) and returns the B operand.
  auto weights = [&](float (&x)[NT][4], uint32_t (&pb)[NT][2]) {
    bool up = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) up |= fmaxf(x[n][0], x[n][2]) > m_ref[n][0] + kKv8Rise || fmaxf(x[n][1], x[n][3]) > m_ref[n][1] + kKv8Rise;
    if (__any_sync(0xffffffffu, up)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float al[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mm = fmaxf(x[n][e], x[n][2 + e]);
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
          const float mn = mm > m_ref[n][e] + kKv8Rise ? mm : m_ref[n][e];
          al[e] = mn == m_ref[n][e] ? 1.f : exp2f(m_ref[n][e] - mn);       // 0 the first time
          m_ref[n][e] = mn;
          l[n][e] *= al[e];
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) { o[m][n][0] *= al[0]; o[m][n][1] *= al[1]; o[m][n][2] *= al[0]; o[m][n][3] *= al[1]; }
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float m0 = m_ref[n][0] == -INFINITY ? 0.f : m_ref[n][0] - kKv8Bias, m1 = m_ref[n][1] == -INFINITY ? 0.f : m_ref[n][1] - kKv8Bias;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[n][e] = kv8_ex2(x[n][e] - (e & 1 ? m1 : m0));
      const __half2 p0 = __floats2half2_rn(x[n][0], x[n][1]), p1 = __floats2half2_rn(x[n][2], x[n][3]);
      pb[n][0] = transpose8x8(*reinterpret_cast<const uint32_t*>(&p0));
      pb[n][1] = transpose8x8(*reinterpret_cast<const uint32_t*>(&p1));
    }
  };

  uint32_t at_k[2][DH / 64], at_v[4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < DH / 64; ++j) at_k[i][j] = st_place<DH>(g + 8 * i, t * (DH / 64) + j);
#pragma unroll
  for (int e = 0; e < 4; ++e) at_v[e] = kTile + st_place<DH>(2 * t + (e & 1) + 8 * (e >> 1), g * DH / 128) + (DH == 64 ? (g & 1) * 8 : 0);
  int stage = 0;
#pragma unroll 1
  for (int gi = warp; gi < n_groups; gi += kStWarps) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStStages - 2) : "memory");
    __syncwarp();                                 // everybody's copies of this group are there, and the stage before it is read
    const int ahead = gi + (kStStages - 1) * kStWarps;
    request(ahead, stage == 0 ? kStStages - 1 : stage - 1, ahead < n_groups ? __float_as_int(s_group[ahead].w) : 0);
    const unsigned char* tile = ring + stage * (2 * kTile);
    const float4 sc_cur = s_group[gi];
    struct { uint32_t k[2][DH / 16], v[4][DH / 32]; } cur;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < DH / 64; ++j) {
        const uint4 w = *reinterpret_cast<const uint4*>(tile + at_k[i][j]);
        cur.k[i][4 * j] = w.x; cur.k[i][4 * j + 1] = w.y; cur.k[i][4 * j + 2] = w.z; cur.k[i][4 * j + 3] = w.w;
      }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (DH == 128) {
        const uint4 w = *reinterpret_cast<const uint4*>(tile + at_v[e]);
        cur.v[e][0] = w.x; cur.v[e][1] = w.y; cur.v[e][2] = w.z; cur.v[e][3] = w.w;
      } else {
        const uint2 w = *reinterpret_cast<const uint2*>(tile + at_v[e]);
        cur.v[e][0] = w.x; cur.v[e][1] = w.y;
      }
    }
    if (++stage == kStStages) stage = 0;
    float x[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KW; ++ks) {
      uint32_t a0, a1, a2, a3;
      kv8_unpack4<FMT>(cur.k[0][ks], a0, a2);
      kv8_unpack4<FMT>(cur.k[1][ks], a1, a3);
#pragma unroll
      for (int n = 0; n < NT; ++n) mma_f16_16816(x[n], a0, a1, a2, a3, q[n][ks][0], q[n][ks][1]);
    }
    const int left = k1 - (k0 + 16 * gi);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float c0 = crow[n][0] * sc_cur.x, c1 = crow[n][1] * sc_cur.x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[n][e] = fmaf(x[n][e], e & 1 ? c1 : c0, sc_cur.y);
    }
    if (left < 16) {          // keys behind the end: no weight, and whatever their bytes hold reads as zero
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
          if (g + 8 * (e >> 1) >= left) x[n][e] = -INFINITY;
#pragma unroll
        for (int w = 0; w < DH / 32; ++w)
          if (2 * t + (e & 1) + 8 * (e >> 1) >= left) cur.v[e][w] = 0u;
      }
    }
    uint32_t pb[NT][2];
    weights(x, pb);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      l[n][0] = fmaf(x[n][0] + x[n][2], sc_cur.z, l[n][0]);
      l[n][1] = fmaf(x[n][1] + x[n][3], sc_cur.z, l[n][1]);
    }
#pragma unroll
    for (int w = 0; w < DH / 32; ++w) {
      // bytes j = 4w .. 4w+3 of this lane's d: pairs (key 2t, key 2t + 1) and (2t + 8, 2t + 9)
      uint32_t a00, a01, a02, a03, a10, a11, a12, a13;
      kv8_unpack4<FMT>(__byte_perm(cur.v[0][w], cur.v[1][w], 0x5140), a00, a01);
      kv8_unpack4<FMT>(__byte_perm(cur.v[0][w], cur.v[1][w], 0x7362), a02, a03);
      kv8_unpack4<FMT>(__byte_perm(cur.v[2][w], cur.v[3][w], 0x5140), a10, a11);
      kv8_unpack4<FMT>(__byte_perm(cur.v[2][w], cur.v[3][w], 0x7362), a12, a13);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mma_f16_16816(o[2 * w][n], a00, a01, a10, a11, pb[n][0], pb[n][1]);
        mma_f16_16816(o[2 * w + 1][n], a02, a03, a12, a13, pb[n][0], pb[n][1]);
      }
    }
  }

  // ---- the new rows, 16 at a time, on the last chunk's first warp, each key divided by a power of two
  const int fresh = last && warp == 0 && a.k_new != nullptr ? s.rows : 0;
#pragma unroll 1
  for (int y0 = 0; y0 < fresh; y0 += 16) {
    const bf16* kn = a.k_new + (size_t)((long long)b * a.rows) * a.new_stride + (size_t)h * DH;
    const bf16* vn = a.v_new + (kn - a.k_new);
    float x[NT][4], ksc[2];                      // scale of keys g, g + 8
#pragma unroll
    for (int n = 0; n < NT; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f;
    uint4 raw[2][DH / 32];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool on = y0 + g + 8 * i < s.rows;
#pragma unroll
      for (int e = 0; e < DH / 32; ++e)
        raw[i][e] = on ? *(reinterpret_cast<const uint4*>(kn + (size_t)(y0 + g + 8 * i) * a.new_stride + t * (DH / 4)) + e) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t big = 0;
#pragma unroll
      for (int e = 0; e < DH / 32; ++e) big = kv8_max_finite(big, raw[i][e]);
      big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
      ksc[i] = kv8_pow2(kv8_row_exp(big));
    }
#pragma unroll
    for (int e = 0; e < DH / 32; ++e) {
      uint32_t f0[4], f1[4];
      kv8_bf16x8_to_half(raw[0][e], 1.f / ksc[0], f0);
      kv8_bf16x8_to_half(raw[1][e], 1.f / ksc[1], f1);
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          mma_f16_16816(x[n], f0[2 * w], f1[2 * w], f0[2 * w + 1], f1[2 * w + 1], q[n][2 * e + w][0], q[n][2 * e + w][1]);
    }
    uint32_t vf[4][DH / 16];                     // fp16 pairs of this lane's DH/8 values of its four keys
    int ev[4];
    bool odd = false;                            // a value that is not finite
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int y = y0 + 2 * t + (e & 1) + 8 * (e >> 1);
      const bool on = y < s.rows;
      uint4 rv[DH / 64];
      uint32_t big = 0;
#pragma unroll
      for (int w = 0; w < DH / 64; ++w) {
        rv[w] = on ? *(reinterpret_cast<const uint4*>(vn + (size_t)y * a.new_stride + g * (DH / 8)) + w) : make_uint4(0u, 0u, 0u, 0u);
        odd |= kv8_zero_non_finite(rv[w]);
        big = kv8_max_finite(big, rv[w]);
      }
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, d));
      ev[e] = kv8_row_exp(big) - kv8_lift(FMT);
#pragma unroll
      for (int w = 0; w < DH / 64; ++w) {
        uint32_t f[4];
        kv8_bf16x8_to_half(rv[w], kv8_pow2(-ev[e]), f);
#pragma unroll
        for (int d = 0; d < 4; ++d) vf[e][4 * w + d] = f[d];
      }
    }
    int evk[2];                                  // of keys g, g + 8: the lanes g / 2 have them
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e0 = __shfl_sync(0xffffffffu, ev[2 * i], g >> 1), e1 = __shfl_sync(0xffffffffu, ev[2 * i + 1], g >> 1);
      evk[i] = g & 1 ? e1 : e0;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 2 * t + (e & 1) + 8 * n, y = y0 + g + 8 * (e >> 1);
        const bool see = i < Nv && y < s.rows && kv8_sees(a, b, i / a.G, y);
        x[n][e] = see ? fmaf(x[n][e], crow[n][e & 1] * ksc[e >> 1], (float)evk[e >> 1]) : -INFINITY;
      }
    uint32_t pb[NT][2];
    weights(x, pb);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) l[n][e & 1] = fmaf(x[n][e] * kKv8Unbias, kv8_pow2(-evk[e >> 1]), l[n][e & 1]);
#pragma unroll
    for (int m = 0; m < MT; ++m) {               // d = g * DH/8 + 2m (A rows g) and + 2m + 1 (rows g + 8)
      const uint32_t w0 = vf[0][m], w1 = vf[1][m], w2 = vf[2][m], w3 = vf[3][m];
#pragma unroll
      for (int n = 0; n < NT; ++n)
        mma_f16_16816(o[m][n], __byte_perm(w0, w1, 0x5410), __byte_perm(w0, w1, 0x7632), __byte_perm(w2, w3, 0x5410),
                      __byte_perm(w2, w3, 0x7632), pb[n][0], pb[n][1]);
    }
    if (__any_sync(0xffffffffu, odd)) {          // values that are not finite reach exactly the rows that see them
#pragma unroll 1
      for (int y = y0; y < min(s.rows, y0 + 16); ++y)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int i = 2 * t + e + 8 * n;
            if (i >= Nv || !kv8_sees(a, b, i / a.G, y)) continue;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int d = 0; d < 2; ++d) {
                const float v = __bfloat162float(vn[(size_t)y * a.new_stride + g * (DH / 8) + 2 * m + d]);
                if (!isfinite(v)) o[m][n][2 * d + e] += v;
              }
          }
    }
    if (NT <= 2) break;                            // (16 rows at most: no loop)
  }

  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();                                // the rings are done with: O takes their place
  // ---- the warps' parts (O without its bias from here on), joined in warp order
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
      if (g == 0) { s_m[warp][2 * t + e + 8 * n] = m_ref[n][e]; s_l[warp][2 * t + e + 8 * n] = l[n][e]; }
    }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *reinterpret_cast<float2*>(&s_o[warp][2 * t + e + 8 * n][g * (DH / 8) + 2 * m]) = make_float2(o[m][n][e] * kKv8Unbias, o[m][n][2 + e] * kKv8Unbias);
  __syncthreads();
#pragma unroll 1
  for (int x = threadIdx.x; x < N * (DH / 4); x += kStWarps * 32) {
    const int i = x / (DH / 4), c4 = x % (DH / 4);
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < kStWarps; ++w) M = fmaxf(M, s_m[w][i]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kStWarps; ++w) {
      if (s_l[w][i] == 0.f) continue;            // no key in this warp
      const float f = exp2f(s_m[w][i] - M);
      const float4 v = *reinterpret_cast<const float4*>(&s_o[w][i][c4 * 4]);
      L += s_l[w][i] * f;
      acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f;
    }
    if (sp.n == 1) {
      kv8_store_row(a, b, h, i, i < Nv, L, c4, acc);
    } else {
      const size_t part = ((size_t)(b * a.c.hkv + h) * plan.max_chunks + chunk_id) * NR + i;
      DART_CHECK(i < NR && chunk_id < plan.max_chunks, a.status) {
        *reinterpret_cast<float4*>(plan.o_part + part * DH + c4 * 4) = acc;
        if (c4 == 0) *reinterpret_cast<float2*>(plan.ml_part + part * 2) = make_float2(M, L);
      }
    }
  }
}

// ---- the join ---------------------------------------------------------------------------------------------------------
// WPR warps per row, partials in a fixed order.  Sequences that fit one chunk were finished by their only CTA.  What bounds
// it is one row's chain of reads, so eight partials are read at a time: with 54 partials a single warp and two dependent rounds
// took 38 us, eight warps and one round take about 4.
template <int WPR>
__global__ void __launch_bounds__(256) kv8_combine_kernel(const __grid_constant__ Kv8AttnArgs a, const Kv8Plan plan) {
  constexpr int kRows = 8 / WPR;
  __shared__ float s_M[8], s_L[8];
  __shared__ __align__(16) float4 s_o[8][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, dh = a.c.dh;
  const int i = blockIdx.x * kRows + warp / WPR, w = warp % WPR, h = blockIdx.y, b = blockIdx.z;
  const Kv8Seq s = kv8_seq(a, b, false);
  const int N = a.rows * a.G, Nv = s.rows * a.G;
  int n = 0;
  size_t part0 = 0, step = 128;
  if (i < N) {
    if (plan.umma) {
      const int tile = i >> 7;
      n = kv8_tiles(a, plan, s, tile).split.n;
      part0 = ((size_t)((b * a.c.hkv + h) * plan.n_tiles + tile) * plan.max_chunks) * 128 + (i & 127);
    } else {
      n = kv8_split_keys(s.len, plan.chunk).n;
      step = (N + 7) / 8 * 8;
      part0 = ((size_t)(b * a.c.hkv + h) * plan.max_chunks) * step + i;
    }
  }
  pdl_wait();
  if (WPR == 1 ? n <= 1 : false) return;
  float M = -INFINITY, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (n > 1) {
    const int c4 = min(lane, dh / 4 - 1);
#pragma unroll 1
    for (int c0 = w; c0 < n; c0 += 8 * WPR) {      // eight partials at a time, all their reads in flight together
      float2 ml[8];
      float4 v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const size_t p = part0 + min(c0 + q * WPR, n - 1) * step;
        ml[q] = *reinterpret_cast<const float2*>(plan.ml_part + p * 2);
        v[q] = *reinterpret_cast<const float4*>(plan.o_part + p * dh + c4 * 4);
      }
      float mn = M;
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (c0 + q * WPR < n) mn = fmaxf(mn, ml[q].x);
      const float up = M == mn ? 1.f : exp2f(M - mn);      // 0 the first time
      M = mn;
      L *= up;
      acc.x *= up; acc.y *= up; acc.z *= up; acc.w *= up;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (c0 + q * WPR >= n || ml[q].y == 0.f) continue;      // no key in this chunk
        const float f = exp2f(ml[q].x - M);
        L += ml[q].y * f;
        acc.x += v[q].x * f; acc.y += v[q].y * f; acc.z += v[q].z * f; acc.w += v[q].w * f;
      }
    }
  }
  if (WPR > 1) {
    if (lane == 0) { s_M[warp] = M; s_L[warp] = L; }
    s_o[warp][lane] = acc;
    __syncthreads();
    if (w != 0 || n <= 1) return;
    M = -INFINITY;
#pragma unroll
    for (int q = 0; q < WPR; ++q) M = fmaxf(M, s_M[q]);
    L = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int q = 0; q < WPR; ++q) {
      if (s_L[q] == 0.f) continue;
      const float f = exp2f(s_M[q] - M);
      const float4 v = s_o[q][lane];
      L += s_L[q] * f;
      acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f;
    }
  }
  if (lane * 4 < dh) kv8_store_row(a, b, h, i, i < Nv, L, lane, acc);
}

// ---- planning ---------------------------------------------------------------------------------------------------------
namespace {

// Keys a CTA of the streaming kernel takes.  With few (batch entry, KV head) pairs one wave of CTAs shares the
// longest sequence evenly; with many, whose lengths differ in a way only the device knows, two waves of shorter parts even
// them out.  (One wave / two / four, us, 64 sequences of 512 to 8192 keys, longest first: 100.6 / 96.9 / 101.0, shortest first
// 107 / 103 / 103, shuffled 106 / 104 / 103; all of 4352: 123 / 110.5 / 106.5; 16 of 8192: 66 / 59 / 61; one of 16384 among 63 of
// 1024: 95 / 94 / 66.)  All of it by max_len, not by the lengths, so a loose bound costs: 64 sequences with a bound of four times
// the longest 97 -> 101.6, one of 4096 keys with a bound of 131072 12.2 -> 21.1.  At least 512 keys, so that a CTA's start (page
// ids, queries, the join) stays a small part.
constexpr int kStMinChunk = 512, kStMaxChunk = 8192;
int round128(long long x) { return (int)((x + 127) / 128 * 128); }

Kv8Plan make_plan(const Kv8AttnArgs& a, void* workspace) {
  Kv8Plan p;
  memset(&p, 0, sizeof(p));
  p.umma = a.rows * a.G > kv8_stream_rows(a.c.dh) ? 1 : 0;
  size_t rows, most;                 // partial rows of this call; of any call with a smaller max_len
  if (!p.umma) {
    const long long pairs = (long long)a.batch * a.c.hkv, part = (a.rows * a.G + 7) / 8 * 8;      // rows of a partial result
    const long long slots = 148 * kv8_stream_ctas(a.c.dh, (a.rows * a.G + 7) / 8), units = pairs * 4 <= slots ? slots : 2 * slots;
    const int parts = (int)((units + pairs - 1) / pairs);               // CTAs per pair if every sequence were the longest
    const int longest = round128(((long long)a.max_len + 65534) / 65535);   // the grid's third dimension
    int chunk = round128(((long long)a.max_len + parts - 1) / parts);
    chunk = chunk < kStMinChunk ? kStMinChunk : chunk > kStMaxChunk ? kStMaxChunk : chunk;
    p.chunk = chunk > longest ? chunk : longest;
    p.max_chunks = kv8_split(a.max_len, p.chunk, 128).n;
    p.n_tiles = 1;
    const long long by_min = ((long long)a.max_len + kStMinChunk - 1) / kStMinChunk, by_max = ((long long)a.max_len + kStMaxChunk - 1) / kStMaxChunk;
    const long long bound = parts > by_max ? parts : by_max;
    most = (size_t)pairs * part * (size_t)(by_min < bound ? by_min : bound);
    rows = (size_t)pairs * part * p.max_chunks;
    if (a.max_len <= kStMinChunk) most = 0;
  } else {
    kv8_umma_plan(a, p);
    rows = (size_t)a.batch * a.c.hkv * p.n_tiles * 128 * p.max_chunks;
    most = p.bytes;
  }
  if (p.max_chunks == 1) rows = 0;
  p.o_part = static_cast<float*>(workspace);
  p.ml_part = p.o_part + rows * a.c.dh;
  p.bytes = 16 + (most > rows ? most : rows) * (a.c.dh + 2) * sizeof(float);
  return p;
}

template <int FMT, int DH, int NT>
cudaError_t launch_stream(const Kv8AttnArgs& a, const Kv8Plan& p, cudaStream_t st) {
  const auto kernel = kv8_attn_stream_kernel<FMT, DH, NT>;
  const size_t most = st_body<DH, NT>() + 32768 / 16 * sizeof(float4);           // with the longest chunk there can be
  const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), most);
  if (e != cudaSuccess) return e;
  prefer_max_shared(reinterpret_cast<const void*>(kernel));
  kernel<<<dim3(a.c.hkv, a.batch, p.max_chunks), kStWarps * 32, st_body<DH, NT>() + p.chunk / 16 * sizeof(float4), st>>>(a, p);
  return cudaGetLastError();
}
template <int FMT, int DH>
cudaError_t launch_stream_rows(const Kv8AttnArgs& a, const Kv8Plan& p, cudaStream_t st) {
  const int n = (a.rows * a.G + 7) / 8;
  if constexpr (kv8_stream_rows(DH) > 24)
    if (n == 4) return launch_stream<FMT, DH, 4>(a, p, st);
  return n == 1 ? launch_stream<FMT, DH, 1>(a, p, st) : n == 2 ? launch_stream<FMT, DH, 2>(a, p, st) : launch_stream<FMT, DH, 3>(a, p, st);
}

}  // namespace

Kv8Plan kv8_attention_plan(const Kv8AttnArgs& a) { return make_plan(a, nullptr); }
size_t kv8_attention_workspace(const Kv8AttnArgs& a) { return make_plan(a, nullptr).bytes; }

cudaError_t launch_kv8_attention(const Kv8AttnArgs& a, void* workspace, int spin, int withhold, cudaStream_t st) {
  Kv8Plan p = make_plan(a, workspace);
  p.spin = spin;
  p.withhold = withhold;
  cudaError_t e;
  if (p.umma)
    e = launch_kv8_attn_umma(a, p, st);
  else if (a.c.format == KV8_E4M3)
    e = a.c.dh == 128 ? launch_stream_rows<KV8_E4M3, 128>(a, p, st) : launch_stream_rows<KV8_E4M3, 64>(a, p, st);
  else
    e = a.c.dh == 128 ? launch_stream_rows<KV8_INT8, 128>(a, p, st) : launch_stream_rows<KV8_INT8, 64>(a, p, st);
  if (e != cudaSuccess || p.max_chunks == 1) return e;
  const int rows = a.rows * a.G;
  // eight warps a row where there are few rows and many partials; elsewhere the rows fill the GPU by themselves
  if (p.max_chunks > 4 && (long long)rows * a.c.hkv * a.batch <= 148 * 8) return launch_pdl(kv8_combine_kernel<8>, dim3(rows, a.c.hkv, a.batch), dim3(256), 0, st, a, p);
  return launch_pdl(kv8_combine_kernel<1>, dim3((rows + 7) / 8, a.c.hkv, a.batch), dim3(256), 0, st, a, p);
}

}  // namespace dart
