// Attention over the paged 8-bit cache: the plain kernel.  One block per (row, query head, batch entry); four warps take
// the visible keys in turn, each with an online softmax of its own, merged at the end.
#include "kv8.cuh"

namespace dart {

__global__ void __launch_bounds__(128) kv8_attn_plain_kernel(const __grid_constant__ Kv8AttnArgs a) {
  const int r = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, h = hq / a.G, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int dh = a.c.dh, per = dh / 32;
  const Kv8Seq s = kv8_seq(a, b, threadIdx.x == 0);
  __shared__ float sm_m[4], sm_l[4], sm_o[4][128];
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  const bf16* qp = a.q + (size_t)(b * (long long)a.rows + r) * a.q_stride + (size_t)hq * dh;
  for (int e = 0; e < per; ++e) q[e] = __bfloat162float(qp[lane * per + e]) * a.scale_log2e;
  const int n_new = (a.k_new != nullptr && r < s.rows) ? s.rows : 0;
  const int total = r < s.rows ? s.len + n_new : 0;
  for (int t = warp; t < total; t += 4) {
    float k[4], v[4];
    if (t < s.len) {
      const int page = kv8_page(a, s.slot, t >> a.c.pt_log2);
      const size_t ph = (size_t)page * a.c.hkv + h, off = (ph * a.c.pt + (t & (a.c.pt - 1))) * dh + lane * per;
      for (int e = 0; e < per; ++e) {
        if (a.c.format == KV8_E4M3) {
          k[e] = __half2float(__half(__nv_cvt_fp8_to_halfraw(a.c.k[off + e], __NV_E4M3)));
          v[e] = __half2float(__half(__nv_cvt_fp8_to_halfraw(a.c.v[off + e], __NV_E4M3)));
        } else {
          k[e] = (float)(int8_t)a.c.k[off + e];
          v[e] = (float)(int8_t)a.c.v[off + e];
        }
        k[e] *= a.c.ks[ph];
        v[e] *= a.c.vs[ph];
      }
    } else {
      const int y = t - s.len;
      const bool see = a.mask != nullptr ? a.mask[((size_t)b * a.rows + r) * a.rows + y] != 0 : y <= r;
      if (!see) continue;
      const size_t off = (size_t)(b * (long long)a.rows + y) * a.new_stride + (size_t)h * dh + lane * per;
      for (int e = 0; e < per; ++e) { k[e] = __bfloat162float(a.k_new[off + e]); v[e] = __bfloat162float(a.v_new[off + e]); }
    }
    float x = 0.f;
    for (int e = 0; e < per; ++e) x += q[e] * k[e];
    x = warp_sum(x);
    const float mn = fmaxf(m, x), al = exp2f(m - mn), p = exp2f(x - mn);
    m = mn;
    l = l * al + p;
    for (int e = 0; e < per; ++e) o[e] = o[e] * al + p * v[e];
  }
  if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
  for (int e = 0; e < per; ++e) sm_o[warp][lane * per + e] = o[e];
  __syncthreads();
  if ((int)threadIdx.x >= dh) return;
  const float M = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
  float L = 0.f, O = 0.f;
  for (int w = 0; w < 4; ++w) {
    if (sm_l[w] == 0.f) continue;      // no key (a NaN score leaves m alone and l NaN)
    const float f = exp2f(sm_m[w] - M);
    L += sm_l[w] * f;
    O += sm_o[w][threadIdx.x] * f;
  }
  a.out[((size_t)(b * (long long)a.rows + r) * a.hq + hq) * dh + threadIdx.x] = __float2bfloat16_rn(L == 0.f ? 0.f : O / L);
}

size_t kv8_attention_workspace(const Kv8AttnArgs&) { return 16; }

cudaError_t launch_kv8_attention(const Kv8AttnArgs& a, void*, cudaStream_t st) {
  kv8_attn_plain_kernel<<<dim3(a.rows, a.hq, a.batch), 128, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace dart
