// Attention over the paged 8-bit cache for many rows (draft trees, prompt chunks, wide head groups), on tcgen05.
// The mathematics is that of kv8_attn.cu; rows r * G + g of a KV head's group form tiles of 128, keys come in steps of 128.
//
// A CTA runs two softmax / MMA pipelines that hide one another's latencies:
//   * two row tiles: both pipelines use every key step, so a step's codes are fetched and converted once for 256 rows;
//   * one row tile (up to 128 rows, or an odd last tile): the key steps alternate between the pipelines, whose results are
//     joined at the end.
// Data path of a step: the producer warp copies the codes of 64 keys at a time (a page, several, or half of one:
// cp.async.bulk, the pages lie where the table says) into a ring of shared-memory slots; four converter warps turn
// them into fp16 (exact) K and V tiles in the 128-byte-swizzle operand layout, two buffers each, and write every key's
// scales beside them; an issuer thread per pipeline runs
//   S = Q K^T   tcgen05.mma 128 x 128, k = DH, Q and K from shared memory, S fp32 in tensor memory
//   O += P V    tcgen05.mma 128 x DH, k = 64 twice, P (fp16) from TENSOR memory, V as stored ([keys][DH], MN-major B)
// and four softmax warps per pipeline (a row per thread) read S 64 columns at a time, and write P over the columns of S
// they have already read.  P in tensor memory instead of shared memory: the MMAs are bound by shared-memory operand reads
// here (128 x 128 x 16 reads 8 KB = 64 cycles' worth from two shared operands, 4 KB with one in tensor memory), and the
// room is needed for the converted tiles.
// New rows are read by the converters themselves, each key divided by its own power of two; a value that is not finite is
// kept out of the product (0 weight times NaN would reach rows that do not see it) and added at the end to the rows that do.
// Every wait is bounded.
#include "kv8.cuh"
#include "umma.cuh"
#include "umma_attn.cuh"

namespace dart {

using namespace umma;

constexpr int kKuThreads = 512;      // warps 0: producer, 1 and 3: MMA issuers, 2: tensor memory; 4-7, 8-11: softmax; 12-15: converters
constexpr int kKuPairSlots = 3, kKuSingleSlots = 7;     // 64-key code slots: what shared memory leaves
constexpr int kKuBad = 4096 / 32;

template <int DH>
struct KuLayout {
  static constexpr int tile = 128 * DH * 2;                       // Q, K and V tiles in fp16
  static constexpr int slot = 64 * DH;                            // codes of 64 keys
  static constexpr size_t smem = 1024 + (size_t)(6 * tile + kKuPairSlots * slot > 5 * tile + kKuSingleSlots * slot
                                                     ? 6 * tile + kKuPairSlots * slot : 5 * tile + kKuSingleSlots * slot);
};

// Instruction descriptor: fp16 A and B, fp32 D.
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N) { return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24); }

// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void mma_f16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(tmem_d),
               "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
               : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
      "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
      "r"(r[31])
      : "memory");
}
// Two fp32 operations in one instruction.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float x, float y) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// Registers per thread of a warpgroup from here on (the kernel is launched with 128): softmax 152 x 256 threads,
// converters 104 x 128, the rest 104 x 128, together the 65536 the block was launched with.
template <int N>
__device__ __forceinline__ void reg_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void reg_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src),
               "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

template <int FMT, int DH>
__global__ void __launch_bounds__(kKuThreads, 1) kv8_attn_umma_kernel(const __grid_constant__ Kv8AttnArgs a, const Kv8Plan plan) {
  using Ly = KuLayout<DH>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ uint64_t q_full[2], c_full[kKuSingleSlots], c_empty[kKuSingleSlots], k_full[2], k_empty[2], v_full[2], v_empty[2];
  __shared__ uint64_t sc_full[2], s_full[2][2], p_full[2][2], pv_done[2][2];
  __shared__ __align__(16) float4 s_sc[2][128];        // per key of a step: scale of k, log2 and reciprocal of v's
  __shared__ float2 s_ml[2][128];
  __shared__ uint32_t s_bad[kKuBad];                   // new rows with a v value that is not finite
  __shared__ uint32_t tmem_base;
  __shared__ int abort_flag, any_bad;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = blockIdx.x, b = blockIdx.y;
  const Kv8Seq s = kv8_seq(a, b, tid == 0 && h == 0 && blockIdx.z == 0);
  // unit -> (group of row tiles, chunk): chunk-major, so that the full chunks of all sequences start first
  const int groups = (plan.n_tiles + 1) / 2;
  const int group = (int)blockIdx.z % groups, chunk_id = (int)blockIdx.z / groups;
  const Kv8Tiles tl = kv8_tiles(a, plan, s, 2 * group);
  if (chunk_id >= tl.split.n) return;
  const int j0 = chunk_id * tl.split.per, n = min(tl.steps - j0, tl.split.per);     // this CTA's steps j0 .. j0 + n - 1
  const int N = a.rows * a.G, Nv = s.rows * a.G;

  if (n <= 0) {                    // no keys at all: zero rows
    for (int e = tid; e < tl.count * 128 * (DH / 4); e += kKuThreads) {
      const int i = tl.first * 128 + e / (DH / 4);
      if (i < N) kv8_store_row(a, b, h, i, false, 0.f, e % (DH / 4), make_float4(0.f, 0.f, 0.f, 0.f));
    }
    return;
  }
  const bool pair = tl.count == 2;
  const int n_slots = pair ? kKuPairSlots : kKuSingleSlots;
  const int n_cached = max(0, min(n, tl.cached - j0));            // the first of this CTA's steps read the cache
  uint8_t* sQ = sm;
  uint8_t* sK = sQ + (pair ? 2 : 1) * Ly::tile;
  uint8_t* sV = sK + 2 * Ly::tile;
  uint8_t* sC = sV + 2 * Ly::tile;

  if (tid == 0) {
    for (int i = 0; i < kKuSingleSlots; ++i) { mbar_init(&c_full[i], 1); mbar_init(&c_empty[i], 4); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 4);
      mbar_init(&k_full[i], 4); mbar_init(&k_empty[i], pair ? 2 : 1);      // one release per pipeline that reads the buffer
      mbar_init(&v_full[i], 4); mbar_init(&v_empty[i], pair ? 2 : 1);
      mbar_init(&sc_full[i], 4);
      for (int hf = 0; hf < 2; ++hf) { mbar_init(&s_full[i][hf], 1); mbar_init(&p_full[i][hf], 4); mbar_init(&pv_done[i][hf], 1); }
    }
    abort_flag = 0;
    any_bad = 0;
    fence_barrier_init();
  }
  if (tid < kKuBad) s_bad[tid] = 0u;
  if (warp == 2) tmem_alloc(&tmem_base, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;      // pipeline p: columns 256 p + {0, 64}: S of a step's halves, each under its P; 256 p + 128: O

  // pipeline p's i-th step: every step with two row tiles, every other one with a single tile
  auto step_of = [&](int p, int i) { return pair ? i : 2 * i + p; };
  auto steps_of = [&](int p) { return pair ? n : (n + 1 - p) >> 1; };

  if (warp < 4) {
   reg_dec<104>();
   if (warp == 0) {
    // ---- producer: 64-key slots in the order K low, K high, V low, V high of every cached step
    const int pages = 64 >> a.c.pt_log2 > 0 ? 64 >> a.c.pt_log2 : 1, toks = 64 / pages;     // copies per slot, tokens each
    const int total = 4 * n_cached;
    auto page_at = [&](int t) -> int {       // this lane's page of slot t, -1: none
      const int key = ((j0 + (t >> 2)) << 7) + ((t & 1) << 6) + lane * toks;
      return t < total && lane < pages && key < s.len ? kv8_page(a, s.slot, key >> a.c.pt_log2) : -1;
    };
    int page = page_at(0), issued = 0, st = 0, use = 0;
    for (int t = 0; t < total; ++t) {
      const int page_next = page_at(t + 1);
      if (use > 0 && !ta_wait(&c_empty[st], (use - 1) & 1, &abort_flag)) break;
      const int active = __popc(__ballot_sync(0xffffffffu, page >= 0));
      if (lane == 0) mbar_expect_tx(&c_full[st], active * toks * DH);      // 0 bytes: the slot lies behind the end, the phase completes
      __syncwarp();
      if (page >= 0) {
        const int key = ((j0 + (t >> 2)) << 7) + ((t & 1) << 6) + lane * toks;
        const uint8_t* src = (t & 2 ? a.c.v : a.c.k) + (((size_t)page * a.c.hkv + h) * a.c.pt + (key & (a.c.pt - 1))) * DH;
        bulk_load(sC + st * Ly::slot + lane * toks * DH, src, toks * DH, &c_full[st]);
      }
      issued = t + 1;
      page = page_next;
      if (++st == n_slots) { st = 0; ++use; }
    }
    if (abort_flag)                  // leave no copy in flight behind
      for (int t = max(0, issued - n_slots); t < issued; ++t)
        for (int it = 0; it < 1000000 && !mbar_test_wait(&c_full[t % n_slots], (t / n_slots) & 1); ++it) {}
   } else if (warp == 2) {
    // ---- the keys' scales: one set per key, four keys (of one page) per lane; a step ahead of their use
    auto scales = [&](int j) {
      const int key = ((j0 + j) << 7) + lane * 4;
      float2 sc = make_float2(0.f, 1.f);
      if (j < n_cached && key < s.len) {
        const size_t ph = (size_t)kv8_page(a, s.slot, key >> a.c.pt_log2) * a.c.hkv + h;
        sc = make_float2(a.c.ks[ph], a.c.vs[ph]);
      }
      return sc;
    };
    float2 sc = scales(0);
    for (int j = 0; j < n_cached; ++j) {
      const int buf = j & 1, use = j >> 1;
      const float2 next = scales(j + 1);
      const float sv = fmaxf(sc.y, kv8_pow2(-100));
      const float4 v = make_float4(sc.x, __log2f(sv), 1.f / sv, 0.f);
      if (use > 0 && !ta_wait(&v_empty[buf], (use - 1) & 1, &abort_flag)) break;
#pragma unroll
      for (int q = 0; q < 4; ++q) s_sc[buf][lane * 4 + q] = v;
      __syncwarp();
      if (lane < 4) mbar_arrive(&sc_full[buf]);      // (new rows: one arrival per converter warp)
      sc = next;
    }
   } else if (lane == 0) {
    // ---- MMA issuer of pipeline p
    const int p = warp >> 1, np = steps_of(p), nh = 2 * np;       // half steps of 64 keys
    constexpr uint32_t idesc_s = idesc_f16(128, 64), idesc_o = idesc_f16(128, DH) | kIdescBMnMajor;
    const uint32_t qa = smem_u32(sQ + (pair ? p : 0) * Ly::tile);
    const uint32_t tS = tmem + p * 256, tO = tS + 128;
    bool ok = np > 0 && ta_wait(&q_full[pair ? p : 0], 0, &abort_flag);
    auto issue_s = [&](int x) -> bool {      // scores of half step x
      const int j = step_of(p, x >> 1), buf = j & 1, hf = x & 1;
      if (!ta_wait(&k_full[buf], (j >> 1) & 1, &abort_flag)) return false;
      if (x >= 2 && !ta_wait(&pv_done[p][hf], ((x >> 1) - 1) & 1, &abort_flag)) return false;     // P of half x - 2 lies where S goes
      tc_fence_after();
      const uint32_t ka = smem_u32(sK + buf * Ly::tile) + hf * 8192;
#pragma unroll
      for (int k = 0; k < DH / 16; ++k) {
        const uint32_t off = (k >> 2) * 16384 + (k & 3) * 32;
        mma_f16(tS + 64 * hf, desc_sw128(qa + off), desc_sw128(ka + off), idesc_s, k > 0 ? 1u : 0u);
      }
      mma_commit(&s_full[p][hf]);
      if (hf == 1) mma_commit(&k_empty[buf]);
      return true;
    };
    if (ok) ok = issue_s(0) && issue_s(1);
    for (int x = 0; x < nh && ok; ++x) {
      const int j = step_of(p, x >> 1), buf = j & 1, hf = x & 1;
      if (!ta_wait(&v_full[buf], (j >> 1) & 1, &abort_flag) || !ta_wait(&p_full[p][hf], (x >> 1) & 1, &abort_flag)) break;
      tc_fence_after();
      const uint64_t dv = desc_sw128_mn(smem_u32(sV + buf * Ly::tile), 16384);
#pragma unroll
      for (int k = 0; k < 4; ++k) mma_f16_ts(tO, tS + hf * 64 + k * 8, dv + 128 * (hf * 4 + k), idesc_o, (x > 0 || k > 0) ? 1u : 0u);
      mma_commit(&pv_done[p][hf]);
      if (hf == 1) mma_commit(&v_empty[buf]);
      if (x + 2 < nh) ok = issue_s(x + 2);      // while the softmax works on half x + 1
    }
   }
  } else if (warp >= 12) {
    reg_dec<104>();
    // ---- converters: codes (or new rows) to fp16 operand tiles, and the keys' scales
    const int ct = tid - 384, cw = warp - 12;
    int st = 0, round = 0;           // next code slot and how often the ring has gone round
    // the next slot's 64 keys -> rows row0 .. row0 + 63 of an operand tile; rows from `valid` on become zero
    auto convert = [&](uint8_t* tile, int row0, int valid) -> bool {
      if (!ta_wait(&c_full[st], round & 1, &abort_flag)) return false;
      // 16 codes = two operand chunks per thread and access.  The second 64 columns of a row lie 16 KB further on, in
      // the same banks: there the two chunks are stored in the other order, and a quarter warp's stores meet eight different bank groups.
      constexpr int kUnits = DH / 32, kLanes = DH / 16, kRowsPerIt = 128 / kLanes;      // per thread; threads per row
      const uint8_t* src = sC + st * Ly::slot + ct * 16;
      uint4 w[kUnits];
#pragma unroll
      for (int it = 0; it < kUnits; ++it) w[it] = *reinterpret_cast<const uint4*>(src + it * 2048);
      __syncwarp();
      if (lane == 0) mbar_arrive(&c_empty[st]);
      if (++st == n_slots) { st = 0; ++round; }
      const int row1 = row0 + ct / kLanes, c = 2 * (ct % kLanes);      // rows of a thread differ by 16 or 32: one swizzle
      const bool swap = DH == 128 && c >= 8;
      uint8_t* base = tile + (c >> 3) * 16384 + row1 * 128;
      uint8_t* d0 = base + ((((c & 7) + (swap ? 1 : 0)) ^ (row1 & 7)) << 4);
      uint8_t* d1 = base + ((((c & 7) + (swap ? 0 : 1)) ^ (row1 & 7)) << 4);
#pragma unroll
      for (int it = 0; it < kUnits; ++it) {
        const uint32_t x0 = swap ? w[it].z : w[it].x, x1 = swap ? w[it].w : w[it].y, x2 = swap ? w[it].x : w[it].z, x3 = swap ? w[it].y : w[it].w;
        uint4 f, g;
        kv8_unpack4<FMT>(x0, f.x, f.y);
        kv8_unpack4<FMT>(x1, f.z, f.w);
        kv8_unpack4<FMT>(x2, g.x, g.y);
        kv8_unpack4<FMT>(x3, g.z, g.w);
        if (valid < 128 && row1 + it * kRowsPerIt >= valid) f = g = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>(d0 + it * kRowsPerIt * 128) = f;
        *reinterpret_cast<uint4*>(d1 + it * kRowsPerIt * 128) = g;
      }
      return true;
    };
    auto publish = [&](uint64_t* bar) {
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    for (int j = 0; j < n; ++j) {
      const int buf = j & 1, use = j >> 1;
      uint8_t *tk = sK + buf * Ly::tile, *tv = sV + buf * Ly::tile;
      if (use > 0 && !ta_wait(&k_empty[buf], (use - 1) & 1, &abort_flag)) break;
      if (j < n_cached) {
        const int valid = min(128, s.len - ((j0 + j) << 7));
        bool ok = true;
#pragma unroll 1
        for (int q = 0; q < 4 && ok; ++q) {        // K low, K high, V low, V high
          if (q == 2 && use > 0 && !ta_wait(&v_empty[buf], (use - 1) & 1, &abort_flag)) { ok = false; break; }
          ok = convert(q < 2 ? tk : tv, (q & 1) * 64, valid);
          if (ok && (q & 1)) publish(q == 1 ? &k_full[buf] : &v_full[buf]);
        }
        if (!ok) break;
      } else {
        const int y0 = (j0 + j - tl.cached) << 7, y = y0 + ct;          // new row of this thread
        const bool on = y < s.rows;
        const size_t off = (size_t)((long long)b * a.rows + (on ? y : 0)) * a.new_stride + (size_t)h * DH;
        int ek = -64, ev = -64;
#pragma unroll
        for (int is_v = 0; is_v < 2; ++is_v) {
          const uint4* src = reinterpret_cast<const uint4*>((is_v ? a.v_new : a.k_new) + off);
          uint8_t* tile = is_v ? tv : tk;
          uint32_t big = 0;
          bool odd = false;
#pragma unroll 4
          for (int c = 0; c < DH / 8; ++c) {
            uint4 v = on ? src[c] : make_uint4(0u, 0u, 0u, 0u);
            if (is_v) odd |= kv8_zero_non_finite(v);
            big = kv8_max_finite(big, v);
          }
          const int ex = kv8_row_exp(big);
          const float inv = kv8_pow2(-ex);
          if (is_v) ev = ex; else ek = ex;
          if (is_v && use > 0 && !ta_wait(&v_empty[buf], (use - 1) & 1, &abort_flag)) break;
#pragma unroll 4
          for (int c = 0; c < DH / 8; ++c) {      // the row once more, from the cache, instead of 64 registers
            uint4 v = on ? src[c] : make_uint4(0u, 0u, 0u, 0u);
            if (is_v) kv8_zero_non_finite(v);
            uint32_t f[4];
            kv8_bf16x8_to_half(v, inv, f);
            *reinterpret_cast<uint4*>(tile + (c >> 3) * 16384 + ct * 128 + (((c & 7) ^ (ct & 7)) << 4)) = make_uint4(f[0], f[1], f[2], f[3]);
          }
          if (is_v) {
            const uint32_t bits = __ballot_sync(0xffffffffu, odd);
            if (lane == 0 && bits != 0u) { s_bad[(y0 >> 5) + cw] = bits; any_bad = 1; }
            s_sc[buf][ct] = make_float4(kv8_pow2(ek), (float)ev, inv, 0.f);
          }
          publish(is_v ? &v_full[buf] : &k_full[buf]);
        }
        if (abort_flag) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sc_full[buf]);
      }
    }
  } else {
    reg_inc<152>();
    // ---- softmax of pipeline p: thread = row of its tile = tensor-memory lane
    const int p = (warp - 4) >> 2, wq = warp & 3, row = wq * 32 + lane, np = steps_of(p);
    const int i_row = (tl.first + (pair ? p : 0)) * 128 + row;
    const bool on = i_row < Nv;
    const int r = on ? i_row / a.G : 0;
    const uint32_t tS = tmem + ((uint32_t)(wq * 32) << 16) + p * 256, tO = tS + 128;
    float crow;
    {
      const uint4* qp = reinterpret_cast<const uint4*>(a.q + (size_t)((long long)b * a.rows + r) * a.q_stride +
                                                       (size_t)(h * a.G + (on ? i_row % a.G : 0)) * DH);
      uint32_t big = 0;
#pragma unroll
      for (int c = 0; c < DH / 8; ++c) big = kv8_max_finite(big, on ? qp[c] : make_uint4(0u, 0u, 0u, 0u));
      const int ex = kv8_row_exp(big);
      crow = a.scale_log2e * kv8_pow2(ex);
      if (pair || p == 0) {
        const float inv = kv8_pow2(-ex);
        uint8_t* tile = sQ + (pair ? p : 0) * Ly::tile;
#pragma unroll
        for (int c = 0; c < DH / 8; ++c) {
          uint32_t f[4];
          kv8_bf16x8_to_half(on ? qp[c] : make_uint4(0u, 0u, 0u, 0u), inv, f);
          *reinterpret_cast<uint4*>(tile + (c >> 3) * 16384 + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = make_uint4(f[0], f[1], f[2], f[3]);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_full[pair ? p : 0]);
      }
    }
    unsigned long long among = 0;          // tree: the new rows that this row sees
    if (a.mask != nullptr && on)
      for (int y = 0; y < s.rows; ++y)
        if (kv8_sees(a, b, r, y)) among |= 1ull << y;
    float m_ref = -INFINITY, l = 0.f;
    bool ok = true;
    for (int i = 0; i < np && ok; ++i) {
      const int j = step_of(p, i), buf = j & 1;
      if (!ta_wait(&sc_full[buf], (j >> 1) & 1, &abort_flag)) { ok = false; break; }      // the keys' scales
      const bool cached = j < n_cached;
      const int left = s.len - ((j0 + j) << 7);                              // cached keys from this step on
#pragma unroll 1
      for (int hf = 0; hf < 2; ++hf) {
        if (!ta_wait(&s_full[p][hf], i & 1, &abort_flag)) { ok = false; break; }
        tc_fence_after();
        const float4* scp = &s_sc[buf][hf * 64];
        // a new reference rescales what O holds, once the half step before has been added to it
        auto raise = [&](float mt) -> bool {
          float alpha = 1.f;
          if (mt > m_ref + 8.f) {           // also the first visible key (m_ref = -inf)
            alpha = m_ref == -INFINITY ? 1.f : kv8_ex2(m_ref - mt);
            m_ref = mt;
            l *= alpha;
          }
          if ((i > 0 || hf > 0) && __any_sync(0xffffffffu, alpha != 1.f)) {
            if (!ta_wait(&pv_done[p][hf ^ 1], (hf ? i : i - 1) & 1, &abort_flag)) return false;
            tc_fence_after();
#pragma unroll 1
            for (int cb = 0; cb < DH; cb += 16) {
              uint32_t rr[16];
              tmem_ld16(tO + cb, rr);
              tmem_ld_wait();
#pragma unroll
              for (int q = 0; q < 16; ++q) rr[q] = __float_as_uint(__uint_as_float(rr[q]) * alpha);
              tmem_st16(tO + cb, rr);
            }
            tmem_st_wait();
          }
          return true;
        };
        if (cached && left >= 128) {
          // 64 cached keys: one set of scales per 16
          float sv[64], mul[4], add[4], mt = -INFINITY;
          tmem_ld64(tS + hf * 64, sv);
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float4 c = scp[g * 16];
            mul[g] = crow * c.x; add[g] = c.y;
            float x0 = fmaxf(sv[16 * g], sv[16 * g + 1]), x1 = fmaxf(sv[16 * g + 2], sv[16 * g + 3]);
#pragma unroll
            for (int q = 4; q < 16; q += 4) {
              x0 = fmaxf(x0, fmaxf(sv[16 * g + q], sv[16 * g + q + 1]));
              x1 = fmaxf(x1, fmaxf(sv[16 * g + q + 2], sv[16 * g + q + 3]));
            }
            mt = fmaxf(mt, fmaf(fmaxf(x0, x1), mul[g], add[g]));
          }
          ok = raise(mt);
          if (!ok) break;
          const float mu = m_ref == -INFINITY ? 0.f : m_ref;
          uint32_t pk[32];
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float sub = add[g] - mu;
            const f32x2 mul2 = pack2(mul[g], mul[g]), sub2 = pack2(sub, sub);
            f32x2 ls = pack2(0.f, 0.f);
#pragma unroll
            for (int q = 0; q < 16; q += 2) {
              float x0, x1;
              unpack2(fma2(pack2(sv[16 * g + q], sv[16 * g + q + 1]), mul2, sub2), x0, x1);
              const float p0 = kv8_ex2(x0), p1 = kv8_ex2(x1);
              ls = add2(ls, pack2(p0, p1));
              const __half2 v2 = __floats2half2_rn(p0, p1);
              pk[8 * g + q / 2] = *reinterpret_cast<const uint32_t*>(&v2);
            }
            float l0, l1;
            unpack2(ls, l0, l1);
            l = fmaf(l0 + l1, scp[g * 16].z, l);
          }
          tmem_st32(tS + hf * 64, pk);      // over the scores it came from
        } else {
          // the end of the cache, or new rows with a scale per key: 16 columns at a time, twice, in little code
          int hi;                           // last visible column, if they are a prefix
          if (cached) hi = left - 1 - hf * 64;
          else hi = min(r, s.rows - 1) - ((j0 + j - tl.cached) << 7) - hf * 64;
          unsigned long long vis = hi < 0 ? 0ull : hi >= 63 ? ~0ull : (2ull << hi) - 1ull;
          if (!cached && a.mask != nullptr) vis = hf == 0 && j0 + j == tl.cached ? among : 0ull;
          if (!on) vis = 0ull;
          auto scores = [&](int c16, float (&x)[16]) {
            uint32_t rr[16];
            tmem_ld16(tS + hf * 64 + c16, rr);
            tmem_ld_wait();
            const uint32_t v = (uint32_t)(vis >> c16);
#pragma unroll
            for (int q = 0; q < 16; ++q) {
              const float4 c = scp[c16 + q];
              const float y = fmaf(__uint_as_float(rr[q]), crow * c.x, c.y);
              x[q] = (v >> q) & 1u ? y : -INFINITY;
            }
          };
          float x[16], mt = -INFINITY;
#pragma unroll 1
          for (int c16 = 0; c16 < 64; c16 += 16) {
            scores(c16, x);
#pragma unroll
            for (int q = 0; q < 16; ++q) mt = fmaxf(mt, x[q]);
          }
          ok = raise(mt);
          if (!ok) break;
          const float mu = m_ref == -INFINITY ? 0.f : m_ref;
#pragma unroll 1
          for (int c16 = 0; c16 < 64; c16 += 16) {
            scores(c16, x);
            uint32_t pk[8];
#pragma unroll
            for (int q = 0; q < 16; q += 2) {
              const float p0 = kv8_ex2(x[q] - mu), p1 = kv8_ex2(x[q + 1] - mu);
              l = fmaf(p0, scp[c16 + q].z, l);
              l = fmaf(p1, scp[c16 + q + 1].z, l);
              const __half2 v2 = __floats2half2_rn(p0, p1);
              pk[q / 2] = *reinterpret_cast<const uint32_t*>(&v2);
            }
            tmem_st8(tS + hf * 64 + c16 / 2, pk);      // over columns read before: c16 / 2 + 7 < c16 + 16
          }
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[p][hf]);
      }
    }
    if (ok && np > 0) ok = ta_wait(&pv_done[p][1], (np - 1) & 1, &abort_flag);
    s_ml[p][row] = make_float2(m_ref, l);
    tc_fence_before();
    asm volatile("bar.sync 1, 256;" ::: "memory");       // the softmax warps
    tc_fence_after();
    // ---- results: a pipeline's own tile, or the join of the two pipelines of a single tile (half of the columns each)
    if (!abort_flag) {
      const int tile = tl.first + (pair ? p : 0);
      const uint32_t tR = tmem + ((uint32_t)(wq * 32) << 16) + 128;
      const bool two = !pair && n > 1;
      const float2 ml0 = s_ml[pair ? p : 0][row], ml1 = two ? s_ml[1][row] : make_float2(-INFINITY, 0.f);
      const float M = fmaxf(ml0.x, ml1.x);
      const float f0 = ml0.y == 0.f ? 0.f : two ? exp2f(ml0.x - M) : 1.f, f1 = ml1.y == 0.f ? 0.f : exp2f(ml1.x - M);
      const float L = ml0.y * f0 + ml1.y * f1;
      const int c_lo = pair ? 0 : p * (DH / 2), c_hi = pair ? DH : c_lo + DH / 2;
      const size_t part = (((size_t)(b * a.c.hkv + h) * plan.n_tiles + tile) * plan.max_chunks + chunk_id) * 128 + row;
      const bool bad = any_bad != 0;
#pragma unroll 1
      for (int cb = c_lo; cb < c_hi; cb += 16) {
        uint32_t r0[16], r1[16];
        tmem_ld16(tR + (pair ? p * 256 : 0) + cb, r0);
        if (two) tmem_ld16(tR + 256 + cb, r1);
        tmem_ld_wait();
        float o[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          o[q] = f0 == 0.f ? 0.f : __uint_as_float(r0[q]) * f0;
          if (two && f1 != 0.f) o[q] += __uint_as_float(r1[q]) * f1;
        }
        if (i_row < N) {
          if (bad && i_row < Nv) {            // values that are not finite reach exactly the rows that see them
            const int r = i_row / a.G;
            for (int y = 0; y < s.rows; ++y) {
              if (!((s_bad[y >> 5] >> (y & 31)) & 1u) || !kv8_sees(a, b, r, y)) continue;
              const bf16* v = a.v_new + (size_t)((long long)b * a.rows + y) * a.new_stride + (size_t)h * DH + cb;
#pragma unroll
              for (int q = 0; q < 16; ++q) {
                const float x = __bfloat162float(v[q]);
                if (!isfinite(x)) o[q] += x;
              }
            }
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 v = make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
            if (tl.split.n == 1) kv8_store_row(a, b, h, i_row, i_row < Nv, L, cb / 4 + q, v);
            else *reinterpret_cast<float4*>(plan.o_part + part * DH + cb + 4 * q) = v;
          }
        }
        __syncwarp();
      }
      if (tl.split.n > 1 && c_lo == 0 && i_row < N) *reinterpret_cast<float2*>(plan.ml_part + part * 2) = make_float2(M, L);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 2) { tc_fence_after(); tmem_dealloc(tmem, 512); }
  if (abort_flag && tid == 0) kv8_report(a.status, DEV_TIMEOUT);
}

// Key steps of a CTA.  Every CTA costs about six steps' worth of start and end (barriers, queries, the first copies, its
// partial result), a step of one row tile about half a step of two.  Enough CTAs for the GPU at one CTA per SM when there
// are few, several waves' worth when there are many; never fewer than four steps.
void kv8_umma_plan(const Kv8AttnArgs& a, Kv8Plan& p) {
  constexpr int kSms = 148, kMinSteps = 4;
  p.n_tiles = (a.rows * a.G + 127) / 128;
  const long long groups = (p.n_tiles + 1) / 2, cells = groups * a.batch * a.c.hkv;
  const int steps = (int)(((long long)a.max_len + 127) / 128) + (a.k_new != nullptr ? (a.rows + 127) / 128 : 0);
  const long long all = ((long long)a.max_len + 127) / 128 + (a.rows + 127) / 128;       // whether or not there are new rows
  const long long parts = cells >= kSms ? (4 * kSms + cells - 1) / cells : kSms / cells;
  long long chunk = (steps + parts - 1) / parts;
  if (chunk < kMinSteps) chunk = kMinSteps;
  const long long longest = all * groups / 63487 + 1;                                     // the grid's third dimension
  if (chunk < longest) chunk = longest;
  p.chunk = (int)chunk;
  p.max_chunks = kv8_split(steps, p.chunk, 1).n;
  // no shorter max_len needs more parts than this
  long long most = (all + kMinSteps - 1) / kMinSteps;
  if (most > parts) most = parts;
  p.bytes = most > 1 ? (size_t)a.batch * a.c.hkv * p.n_tiles * 128 * (size_t)most : 0;
}

namespace {
template <int FMT, int DH>
cudaError_t launch(const Kv8AttnArgs& a, const Kv8Plan& p, cudaStream_t st) {
  const auto kernel = kv8_attn_umma_kernel<FMT, DH>;
  const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), KuLayout<DH>::smem);
  if (e != cudaSuccess) return e;
  kernel<<<dim3(a.c.hkv, a.batch, (p.n_tiles + 1) / 2 * p.max_chunks), kKuThreads, KuLayout<DH>::smem, st>>>(a, p);
  return cudaGetLastError();
}
}  // namespace

cudaError_t launch_kv8_attn_umma(const Kv8AttnArgs& a, const Kv8Plan& p, cudaStream_t st) {
  if (a.c.format == KV8_E4M3) return a.c.dh == 128 ? launch<KV8_E4M3, 128>(a, p, st) : launch<KV8_E4M3, 64>(a, p, st);
  return a.c.dh == 128 ? launch<KV8_INT8, 128>(a, p, st) : launch<KV8_INT8, 64>(a, p, st);
}

}  // namespace dart
