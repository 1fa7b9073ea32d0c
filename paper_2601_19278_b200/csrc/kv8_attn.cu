// Attention over the paged 8-bit cache (include/dart.h: dart_kv8_attention): planning, the kernel for few rows, the join.
//
//   out[r] = sum_y softmax_y(q[r] . k[y] / sqrt(d)) v[y],   k[y] = s_k * code,  v[y] = s_v * code
//
// Codes of both formats are exact in fp16, and so is a bf16 query or new row once divided by a power of two near its
// largest element, so both products run on fp16 tensor-core instructions with nothing rounded but the weights.  The scales
// never touch the codes: with c = log2(e) / sqrt(d) times the query's power of two, a key of a page with scales s_k, s_v
// enters as
//   x = (c s_k) (q . code) + log2(s_v),     P = 2^(x - m),     l += P / s_v,     O += P code,     out = O / l
// where m follows the largest x (not the largest score): P is the key's weight times its value's scale, at most 2^8, so its
// rounding to fp16 (2^-11, or 2^-25 absolute for weights that do not matter) is relative to what the key contributes,
// however far apart the pages' scales are.  m, l and O are fp32.  New rows are keys with a power-of-two scale of their own.
//
// Rows of all query heads that share a KV head are one matrix (row r, head g of the group -> r * G + g).  Up to 16 such
// rows run on kv8_attn_stream_kernel below: a stream of the cache at memory speed.  More rows run on tcgen05
// (kv8_attn_umma.cu).  A long key axis is split over CTAs; their partial (m, l, O) go through the workspace and
// kv8_combine_kernel joins them.
#include <string.h>

#include "kv8.cuh"

namespace dart {

// ---- few rows ---------------------------------------------------------------------------------------------------------
// What bounds it is the stream of K and V bytes, so nothing is staged: a warp takes 16 keys at a time and every lane loads
// exactly the bytes that its own tensor-core fragments need, 16 (or 8) at a time, one group ahead of the arithmetic.
//   S = Q K^T   mma m16n8k16, rows x keys.  The order of the contraction index is free as long as Q and K agree: lane t of a
//               key's quad takes d = [t * DH/4, (t+1) * DH/4), whole 16-byte words of the key's row.
//   O^T = V^T P^T  the same instruction with d as M: its A operand wants pairs of neighbouring keys, which two bytes of
//               two keys' words give by one byte permutation before the conversion; the scores come out of the first product
//               exactly where the second wants its B operand, so P never leaves its lane.
// m moves only when a score exceeds it by 2^8: the common case has no shuffles at all.
constexpr int kStWarps = 4;

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Bytes of one group of 16 keys that a lane holds: K of keys g and g + 8, V of keys 2t, 2t+1, 2t+8, 2t+9.
template <int DH>
struct Group {
  uint32_t k[2][DH / 16];      // DH/4 bytes each
  uint32_t v[4][DH / 32];      // DH/8 bytes each
};
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&r)[N], const uint8_t* p) {
  static_assert(N == 2 || N % 4 == 0, "");
  if constexpr (N == 2) {
    const uint2 x = __ldg(reinterpret_cast<const uint2*>(p));
    r[0] = x.x; r[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(p) + i);
      r[4 * i] = x.x; r[4 * i + 1] = x.y; r[4 * i + 2] = x.z; r[4 * i + 3] = x.w;
    }
  }
}

// NT = 1: up to 8 rows (the second half of the first product's M is empty), 2: up to 16.
template <int FMT, int DH, int NT>
__global__ void __launch_bounds__(kStWarps * 32, NT == 1 ? 3 : 2) kv8_attn_stream_kernel(const __grid_constant__ Kv8AttnArgs a,
                                                                                        const Kv8Plan plan) {
  constexpr int MT = DH / 16, KW = DH / 16;     // d tiles of the second product; words of a lane's piece of a key
  constexpr int NR = 8 * NT;
  extern __shared__ __align__(16) unsigned char st_smem[];
  int* s_page = reinterpret_cast<int*>(st_smem);                 // [plan.chunk / 16] page of every group of 16 keys
  __shared__ float s_m[kStWarps][NR], s_l[kStWarps][NR];
  __shared__ __align__(16) float s_o[kStWarps][NR][DH];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int h = blockIdx.x, b = blockIdx.y, chunk_id = blockIdx.z;
  const Kv8Seq s = kv8_seq(a, b, threadIdx.x == 0 && h == 0 && chunk_id == 0);
  const int N = a.rows * a.G, Nv = s.rows * a.G;                  // rows of the call, rows that exist
  const Kv8Split sp = kv8_split_keys(s.len, plan.chunk);
  if (chunk_id >= sp.n) return;
  const int k0 = chunk_id * sp.per, k1 = min(s.len, k0 + sp.per);
  const bool last = chunk_id == sp.n - 1;
  for (int i = threadIdx.x; i < (k1 - k0 + 15) / 16; i += kStWarps * 32) s_page[i] = kv8_page(a, s.slot, (k0 + 16 * i) >> a.c.pt_log2);

  // Q fragments: rows g and g + 8, d of this lane in the order of the K words; a power of two brings a row's largest
  // finite element to [1, 2)
  uint32_t qa[KW][2], qb[NT == 2 ? KW : 1][2];
  float crow[NT];
#pragma unroll
  for (int half = 0; half < NT; ++half) {
    const int i = g + 8 * half;
    const bool on = i < Nv;
    const bf16* qp = a.q + (size_t)((long long)b * a.rows + (on ? i / a.G : 0)) * a.q_stride + (size_t)(h * a.G + (on ? i % a.G : 0)) * DH + t * (DH / 4);
    uint4 raw[DH / 32];
    uint32_t big = 0;
#pragma unroll
    for (int e = 0; e < DH / 32; ++e) {
      raw[e] = on ? *(reinterpret_cast<const uint4*>(qp) + e) : make_uint4(0u, 0u, 0u, 0u);
      big = kv8_max_finite(big, raw[e]);
    }
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
    const int ex = kv8_row_exp(big);
    crow[half] = a.scale_log2e * kv8_pow2(ex);
    const float inv = kv8_pow2(-ex);
#pragma unroll
    for (int e = 0; e < DH / 32; ++e) {
      uint32_t f[4];
      kv8_bf16x8_to_half(raw[e], inv, f);
#pragma unroll
      for (int w = 0; w < 2; ++w) {            // word 2e + w of the K piece: d 4 (2e + w) .. + 3
        if (half == 0) { qa[2 * e + w][0] = f[2 * w]; qa[2 * e + w][1] = f[2 * w + 1]; }
        else { qb[NT == 2 ? 2 * e + w : 0][0] = f[2 * w]; qb[NT == 2 ? 2 * e + w : 0][1] = f[2 * w + 1]; }
      }
    }
  }
  __syncthreads();

  float o[MT][NT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) o[m][n][0] = o[m][n][1] = o[m][n][2] = o[m][n][3] = 0.f;
  float m_ref[NT], l[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) { m_ref[n] = -INFINITY; l[n] = 0.f; }

  // x[n][4]: rows g + 8n, keys 2t, 2t+1, 2t+8, 2t+9, scaled, -inf where hidden.  Turns them into P and returns the B operand.
  auto weights = [&](float (&x)[NT][4], uint32_t (&pb)[NT][2]) {
    bool up = false;
    float mt[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      mt[n] = fmaxf(fmaxf(x[n][0], x[n][1]), fmaxf(x[n][2], x[n][3]));
      up |= mt[n] > m_ref[n] + 8.f;
    }
    if (__any_sync(0xffffffffu, up)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float mm = fmaxf(mt[n], __shfl_xor_sync(0xffffffffu, mt[n], 1));
        mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, 2));
        const float mn = mm > m_ref[n] + 8.f ? mm : m_ref[n];
        const float al = mn == m_ref[n] ? 1.f : exp2f(m_ref[n] - mn);       // 0 the first time
        m_ref[n] = mn;
        l[n] *= al;
        const float a0 = __shfl_sync(0xffffffffu, al, 8 * t), a1 = __shfl_sync(0xffffffffu, al, 8 * t + 4);   // rows 2t, 2t + 1
#pragma unroll
        for (int m = 0; m < MT; ++m) { o[m][n][0] *= a0; o[m][n][1] *= a1; o[m][n][2] *= a0; o[m][n][3] *= a1; }
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float mu = m_ref[n] == -INFINITY ? 0.f : m_ref[n];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[n][e] = kv8_ex2(x[n][e] - mu);
      const __half2 p0 = __floats2half2_rn(x[n][0], x[n][1]), p1 = __floats2half2_rn(x[n][2], x[n][3]);
      pb[n][0] = *reinterpret_cast<const uint32_t*>(&p0);
      pb[n][1] = *reinterpret_cast<const uint32_t*>(&p1);
    }
  };

  struct Scales { float k, v; };
  auto load = [&](int gi, Group<DH>& w, Scales& sc) {
    const size_t ph = (size_t)s_page[gi] * a.c.hkv + h;
    const uint8_t* kb = a.c.k + (ph * a.c.pt + ((k0 + 16 * gi) & (a.c.pt - 1))) * DH;
    const uint8_t* vb = a.c.v + (kb - a.c.k);
    sc.k = __ldg(a.c.ks + ph);
    sc.v = __ldg(a.c.vs + ph);
#pragma unroll
    for (int i = 0; i < 2; ++i) load_words(w.k[i], kb + (g + 8 * i) * DH + t * (DH / 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) load_words(w.v[i], vb + (2 * t + (i & 1) + 8 * (i >> 1)) * DH + g * (DH / 8));
  };

  const int n_groups = (k1 - k0 + 15) / 16;
  Group<DH> cur;
  Scales sc_cur = {0.f, 0.f};
  if (warp < n_groups) load(warp, cur, sc_cur);
  for (int gi = warp; gi < n_groups; gi += kStWarps) {
    Group<DH> nxt;
    Scales sc_nxt = {0.f, 0.f};
    if (gi + kStWarps < n_groups) load(gi + kStWarps, nxt, sc_nxt);
    float sc[2][4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KW; ++ks) {
        uint32_t b0, b1;
        kv8_unpack4<FMT>(cur.k[nt][ks], b0, b1);
        mma_f16_16816(sc[nt], qa[ks][0], NT == 2 ? qb[NT == 2 ? ks : 0][0] : 0u, qa[ks][1], NT == 2 ? qb[NT == 2 ? ks : 0][1] : 0u, b0, b1);
      }
    }
    const float sv = fmaxf(sc_cur.v, kv8_pow2(-100)), lsv = __log2f(sv), rsv = 1.f / sv;
    float x[NT][4];
    uint32_t pb[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float cs = crow[n] * sc_cur.k;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[n][e] = fmaf(sc[e >> 1][2 * n + (e & 1)], cs, lsv);
    }
    const int left = k1 - (k0 + 16 * gi);
    if (left < 16) {          // keys behind the end: no weight, and whatever their bytes hold reads as zero
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = 2 * t + (e & 1) + 8 * (e >> 1);
        if (key >= left) {
#pragma unroll
          for (int n = 0; n < NT; ++n) x[n][e] = -INFINITY;
#pragma unroll
          for (int w = 0; w < DH / 32; ++w) cur.v[e][w] = 0u;
        }
      }
    }
    weights(x, pb);
#pragma unroll
    for (int n = 0; n < NT; ++n) l[n] = fmaf((x[n][0] + x[n][1]) + (x[n][2] + x[n][3]), rsv, l[n]);
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
    cur = nxt;
    sc_cur = sc_nxt;
  }

  // ---- the new rows (at most 16): one more group, on the last chunk's first warp
  if (last && warp == 0 && a.k_new != nullptr && s.rows > 0) {
    const size_t nb = (size_t)((long long)b * a.rows) * a.new_stride + (size_t)h * DH;
    float sc[2][4], ksc[4];                      // ksc: scale of keys 2t, 2t+1, 2t+8, 2t+9
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      const int y = g + 8 * nt;
      const bool on = y < s.rows;
      const bf16* kp = a.k_new + nb + (size_t)(on ? y : 0) * a.new_stride + t * (DH / 4);
      uint4 raw[DH / 32];
      uint32_t big = 0;
#pragma unroll
      for (int e = 0; e < DH / 32; ++e) {
        raw[e] = on ? *(reinterpret_cast<const uint4*>(kp) + e) : make_uint4(0u, 0u, 0u, 0u);
        big = kv8_max_finite(big, raw[e]);
      }
      big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
      const int ex = kv8_row_exp(big);
      const float inv = kv8_pow2(-ex);
      sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
#pragma unroll
      for (int e = 0; e < DH / 32; ++e) {
        uint32_t f[4];
        kv8_bf16x8_to_half(raw[e], inv, f);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const int ks = 2 * e + w;
          mma_f16_16816(sc[nt], qa[ks][0], NT == 2 ? qb[NT == 2 ? ks : 0][0] : 0u, qa[ks][1], NT == 2 ? qb[NT == 2 ? ks : 0][1] : 0u, f[2 * w], f[2 * w + 1]);
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) ksc[2 * nt + e] = kv8_pow2(__shfl_sync(0xffffffffu, ex, (2 * t + e) * 4));
    }
    uint32_t vf[4][DH / 16];                     // fp16 pairs of this lane's DH/8 values of its four keys
    float lsv[4], rsv[4];
    bool odd = false;                            // a value that is not finite
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int y = 2 * t + (e & 1) + 8 * (e >> 1);
      const bool on = y < s.rows;
      const bf16* vp = a.v_new + nb + (size_t)(on ? y : 0) * a.new_stride + g * (DH / 8);
      uint4 raw[DH / 64];
      uint32_t big = 0;
#pragma unroll
      for (int w = 0; w < DH / 64; ++w) {
        raw[w] = on ? *(reinterpret_cast<const uint4*>(vp) + w) : make_uint4(0u, 0u, 0u, 0u);
        odd |= kv8_zero_non_finite(raw[w]);
        big = kv8_max_finite(big, raw[w]);
      }
#pragma unroll
      for (int q = 4; q < 32; q <<= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, q));
      const int ex = kv8_row_exp(big);
      const float inv = kv8_pow2(-ex);
      lsv[e] = (float)ex;
      rsv[e] = inv;
#pragma unroll
      for (int w = 0; w < DH / 64; ++w) {
        uint32_t f[4];
        kv8_bf16x8_to_half(raw[w], inv, f);
#pragma unroll
        for (int q = 0; q < 4; ++q) vf[e][4 * w + q] = f[q];
      }
    }
    float x[NT][4];
    uint32_t pb[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = g + 8 * n, y = 2 * t + (e & 1) + 8 * (e >> 1);
        const bool see = i < Nv && y < s.rows && kv8_sees(a, b, i / a.G, y);
        x[n][e] = see ? fmaf(sc[e >> 1][2 * n + (e & 1)], crow[n] * ksc[e], lsv[e]) : -INFINITY;
      }
    weights(x, pb);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) l[n] = fmaf(x[n][e], rsv[e], l[n]);
#pragma unroll
    for (int m = 0; m < MT; ++m) {               // d = g * DH/8 + 2m (A rows g) and + 2m + 1 (rows g + 8)
      const uint32_t w0 = vf[0][m], w1 = vf[1][m], w2 = vf[2][m], w3 = vf[3][m];
#pragma unroll
      for (int n = 0; n < NT; ++n)
        mma_f16_16816(o[m][n], __byte_perm(w0, w1, 0x5410), __byte_perm(w0, w1, 0x7632), __byte_perm(w2, w3, 0x5410),
                      __byte_perm(w2, w3, 0x7632), pb[n][0], pb[n][1]);
    }
    if (__any_sync(0xffffffffu, odd)) {          // values that are not finite reach exactly the rows that see them
      for (int y = 0; y < s.rows; ++y)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int i = 2 * t + e + 8 * n;
            if (i >= Nv || !kv8_sees(a, b, i / a.G, y)) continue;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int q = 0; q < 2; ++q) {
                const float v = __bfloat162float(a.v_new[nb + (size_t)y * a.new_stride + g * (DH / 8) + 2 * m + q]);
                if (!isfinite(v)) o[m][n][2 * q + e] += v;
              }
          }
    }
  }

  // ---- the warps' parts, joined in warp order
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    l[n] += __shfl_xor_sync(0xffffffffu, l[n], 1);
    l[n] += __shfl_xor_sync(0xffffffffu, l[n], 2);
    if (t == 0) { s_m[warp][g + 8 * n] = m_ref[n]; s_l[warp][g + 8 * n] = l[n]; }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *reinterpret_cast<float2*>(&s_o[warp][2 * t + e + 8 * n][g * (DH / 8) + 2 * m]) = make_float2(o[m][n][e], o[m][n][2 + e]);
  __syncthreads();
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
      const size_t part = ((size_t)(b * a.c.hkv + h) * plan.max_chunks + chunk_id) * 16 + i;
      *reinterpret_cast<float4*>(plan.o_part + part * DH + c4 * 4) = acc;
      if (c4 == 0) *reinterpret_cast<float2*>(plan.ml_part + part * 2) = make_float2(M, L);
    }
  }
}

// ---- the join ---------------------------------------------------------------------------------------------------------
// WPR warps per row, partials in a fixed order.  Sequences that fit one chunk were finished by their only CTA.  What bounds
// it is one row's chain of reads: with 54 partials a single warp took 38 us, eight warps take @CMB.
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
  size_t part0 = 0, step = 16;
  if (i < N) {
    if (plan.umma) {
      const int tile = i >> 7;
      n = kv8_tiles(a, plan, s, tile).split.n;
      part0 = ((size_t)((b * a.c.hkv + h) * plan.n_tiles + tile) * plan.max_chunks) * 128 + (i & 127);
      step = 128;
    } else {
      n = kv8_split_keys(s.len, plan.chunk).n;
      part0 = ((size_t)(b * a.c.hkv + h) * plan.max_chunks) * 16 + i;
    }
  }
  pdl_wait();
  if (WPR == 1 ? n <= 1 : false) return;
  float M = -INFINITY, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (n > 1) {
    for (int c = w + lane * WPR; c < n; c += 32 * WPR) M = fmaxf(M, plan.ml_part[(part0 + c * step) * 2]);
    M = warp_max(M);
    const int c4 = min(lane, dh / 4 - 1);
#pragma unroll 4
    for (int c = w; c < n; c += WPR) {
      const size_t p = part0 + c * step;
      const float2 ml = *reinterpret_cast<const float2*>(plan.ml_part + p * 2);
      const float4 v = *reinterpret_cast<const float4*>(plan.o_part + p * dh + c4 * 4);
      if (ml.y == 0.f) continue;      // no key in this chunk
      const float f = exp2f(ml.x - M);
      L += ml.y * f;
      acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f;
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

// Keys a CTA of the streaming kernel takes.  With few (batch entry, KV head) pairs one wave of CTAs (three to an SM)
// shares the longest sequence evenly; with many, whose lengths differ in a way only the device knows, several waves of
// shorter parts even them out.  At least 512 keys, so that a CTA's start (page ids, queries, the join) stays a small part.
constexpr int kStSlots = 148 * 3;
constexpr int kStMinChunk = 512, kStMaxChunk = 8192;
int round128(long long x) { return (int)((x + 127) / 128 * 128); }

Kv8Plan make_plan(const Kv8AttnArgs& a, void* workspace) {
  Kv8Plan p;
  memset(&p, 0, sizeof(p));
  p.umma = a.rows * a.G > 16 ? 1 : 0;
  size_t rows, most;                 // partial rows of this call; of any call with a smaller max_len
  if (!p.umma) {
    const long long pairs = (long long)a.batch * a.c.hkv;
    const long long units = pairs * 4 <= kStSlots ? kStSlots : 6 * kStSlots;
    const int parts = (int)((units + pairs - 1) / pairs);               // CTAs per pair if every sequence were the longest
    const int longest = round128(((long long)a.max_len + 65534) / 65535);   // the grid's third dimension
    int chunk = round128(((long long)a.max_len + parts - 1) / parts);
    chunk = chunk < kStMinChunk ? kStMinChunk : chunk > kStMaxChunk ? kStMaxChunk : chunk;
    p.chunk = chunk > longest ? chunk : longest;
    p.max_chunks = kv8_split(a.max_len, p.chunk, 128).n;
    p.n_tiles = 1;
    const long long by_min = ((long long)a.max_len + kStMinChunk - 1) / kStMinChunk, by_max = ((long long)a.max_len + kStMaxChunk - 1) / kStMaxChunk;
    const long long bound = parts > by_max ? parts : by_max;
    most = (size_t)pairs * 16 * (size_t)(by_min < bound ? by_min : bound);
    rows = (size_t)pairs * 16 * p.max_chunks;
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
  kv8_attn_stream_kernel<FMT, DH, NT><<<dim3(a.c.hkv, a.batch, p.max_chunks), kStWarps * 32, p.chunk / 16 * sizeof(int), st>>>(a, p);
  return cudaGetLastError();
}
template <int FMT, int DH>
cudaError_t launch_stream_rows(const Kv8AttnArgs& a, const Kv8Plan& p, cudaStream_t st) {
  return a.rows * a.G <= 8 ? launch_stream<FMT, DH, 1>(a, p, st) : launch_stream<FMT, DH, 2>(a, p, st);
}

}  // namespace

size_t kv8_attention_workspace(const Kv8AttnArgs& a) { return make_plan(a, nullptr).bytes; }

cudaError_t launch_kv8_attention(const Kv8AttnArgs& a, void* workspace, cudaStream_t st) {
  const Kv8Plan p = make_plan(a, workspace);
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
