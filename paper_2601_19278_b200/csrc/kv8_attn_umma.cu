// Attention over the paged 8-bit cache for many rows (draft trees, prompt chunks, wide head groups), on tcgen05.
// The mathematics is that of kv8_attn.cu; rows r * G + g of a KV head's group form tiles of 128, keys come in steps of 128.
//
// A CTA runs two softmax / MMA pipelines that hide one another's latencies:
//   * two row tiles: both pipelines use every key step, so a step's codes are fetched and converted once for 256 rows;
//   * one row tile (up to 128 rows, or an odd last tile): the key steps alternate between the pipelines, whose results are
//     joined at the end.
// Data path of a step: two producer warps copy the codes of 64 keys at a time (a page, several, or half of one:
// cp.async.bulk, the pages lie where the table says) into rings of shared-memory slots, K and V apart; four converter
// warps for each turn them into fp16 (exact) tiles in the 128-byte-swizzle operand layout, two buffers each, and write
// every key's scales; an issuer warp per pipeline runs, in half steps of 64 keys,
//   S = Q K^T   tcgen05.mma 128 x 64, k = DH, Q and K from shared memory, S fp32 in tensor memory, two buffers
//   O += P V    tcgen05.mma 128 x DH, k = 64, P (fp16) from TENSOR memory, V as stored ([keys][DH], MN-major B)
// and four softmax warps per pipeline (a row per thread) read the scores of a half step and write P over them.  P in tensor
// memory instead of shared memory: operand reads from shared memory are what is scarce, and the room is needed for the
// converted tiles.
// What bounds a step of 256 rows x 128 keys (2.2 us = 1.1 PFLOP/s in all, 0.7 of the bf16 peak): the exponentials (two softmax
// warps share a special-function unit: 1.1 us) and shared memory (operands, codes and converted tiles: about 1.5 us of
// its bandwidth), neither alone: without the exponentials a step takes 1.8, without half of the MMAs 2.1.  What was tried:
// part of the exponentials as polynomials (no faster with two warps to a unit), scores in steps of 128 keys without a second
// buffer (the chain S -> P -> O showed: 2.5), one producer for K and V and half the converters (2.3 to 3.9 while they
// were the slowest role), exponentials interleaved with their sums instead of in phases (3 %).
// A CTA's start and end cost 9 to 13 us (queries to fp16 4, the first scores 3, the result 2) and new rows that only some
// rows see 5 us a step, which is most of a short call.  Code outside the inner loops is kept in loops and short:
// unrolled, it was 100 KB and each CTA waited for its instructions.
// New rows are read by the converters themselves, each key divided by its own power of two; a value that is not finite is
// kept out of the product (0 weight times NaN would reach rows that do not see it) and added at the end to the rows that do.
// Every wait is bounded.  At the 96 registers of the launch the compiler spills 40 to 56 bytes a thread (192 to 204 bytes of loads).
#include "kv8.cuh"
#include "umma.cuh"
#include "umma_attn.cuh"

namespace dart {

using namespace umma;

constexpr int kKuThreads = 640;      // warps 0: producer of K, 1 and 3: MMA issuers, 2: producer of V; 4-7, 8-11: softmax; 12-15, 16-19: converters
constexpr int kKuPairSlots = 2, kKuSingleSlots = 3;     // 64-key code slots of each ring (K, V): what shared memory leaves
constexpr int kKuBad = 4096 / 32;

// Bounded wait in little code (the loop is not unrolled: there are some twenty of them).  try_wait suspends the warp for up to
// 2600 cycles (measured), which leaves the issue slots to the softmax warps beside it (1 % of the kernel's time against
// test_wait, with or without a pause between two looks; with a suspend-time hint, or a look at the clock, 2 to 3 % slower).
// `patience`, in shared memory, is how many tries every wait of the CTA has (plan.spin); the wait that runs out sets it to 0 and
// all roles leave.  (As an argument of the kernel the limit took a register that the softmax warps do not have: 2 % of 16
// trees, 7 % of the prompt chunk.)  A whole warp waits and one answer is every lane's, since what follows has
// instructions that all lanes have to meet; the votes take 0.2 %.
__device__ __forceinline__ bool ku_wait(uint64_t* bar, uint32_t parity, volatile int* patience) {
#pragma unroll 1
  for (int it = 0;; ++it) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    if (__all_sync(0xffffffffu, ok)) return true;
    if (__any_sync(0xffffffffu, it >= *patience)) break;
  }
  *patience = 0;
  return false;
}

// What is not an operand tile or a code slot.
struct KuShared {
  uint64_t q_full[2], c_full[2][kKuSingleSlots], c_empty[2][kKuSingleSlots], k_full[2], k_empty[2], v_full[2], v_empty[2], sc_full[2];
  uint64_t s_full[2][2], p_full[2][2], pv_done[2][2], drained[2];
  float2 sc[2][128];                     // per key of a step: scale of k, log2 of v's
  uint32_t bad[kKuBad];                  // new rows with a v value that is not finite
  uint32_t tmem_base;
  int patience, any_bad;
  int2 issued[2];                        // code slots that the producers of K and V asked for; slots of a ring
};
// Two row tiles: Q, Q, K, K, V, V and two slots a ring; one: Q, K, K, V, V, three slots a ring and the pipelines' (m, l).  With
// DH = 128 the first form is all that a block can have.
template <int DH>
struct KuLayout {
  static constexpr int tile = 128 * DH * 2;                       // an operand tile in fp16
  static constexpr int slot = 64 * DH;                            // codes of 64 keys
  static constexpr int pair = 6 * tile + 2 * kKuPairSlots * slot, single = 5 * tile + 2 * kKuSingleSlots * slot + 2 * 128 * 8;
  static constexpr int body = pair > single ? pair : single;
  static constexpr size_t smem = body + sizeof(KuShared);
  static_assert(smem <= 232448, "a block's shared memory");
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
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Registers per thread of a warpgroup from here on (the kernel is launched with 96): softmax 136 x 256 threads,
// converters 72 x 256, the rest 64 x 128, together the 61440 the block was launched with.
template <int N>
__device__ __forceinline__ void reg_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void reg_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src),
               "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// One bf16 row, divided by a power of two near its largest finite element, as row `row` of an fp16 operand tile.  Through
// the row's own place in shared memory, in loops: code that runs once per CTA has to be short, because instructions that
// are not in the cache cost far more than their work (unrolled, this and the epilogue took 30000 cycles of a 100000-cycle
// CTA).  The largest element ends up in [2^lift, 2^(lift + 1)).  `odd`: values that are not finite become zero, and whether there were any is returned.
template <int DH>
__device__ __forceinline__ bool ku_row_to_operand(const bf16* src, bool on, uint8_t* tile, int row, bool odd, int lift, int& ex) {
  const uint32_t base = smem_u32(tile) + row * 128;
  const int bytes = on ? 16 : 0;         // 0: zeros, nothing is read
#pragma unroll 4
  for (int c = 0; c < DH / 8; ++c)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(base + (c >> 3) * 16384 + (((c & 7) ^ (row & 7)) << 4)), "l"(src + c * 8),
                 "r"(bytes) : "memory");
  asm volatile("cp.async.wait_all;" ::: "memory");
  uint8_t* place = tile + row * 128;
  // the largest |x| bits of both halves of all words, one three-way 16-bit maximum per two words
  uint32_t top = 0;
#pragma unroll 4
  for (int c = 0; c < DH / 8; ++c) {
    const uint4 w = *reinterpret_cast<const uint4*>(place + (c >> 3) * 16384 + (((c & 7) ^ (row & 7)) << 4));
    top = __vimax3_u16x2(top, w.x & 0x7fff7fffu, w.y & 0x7fff7fffu);
    top = __vimax3_u16x2(top, w.z & 0x7fff7fffu, w.w & 0x7fff7fffu);
  }
  uint32_t big = max(top & 0xffffu, top >> 16);
  bool any = false;
  if (big >= 0x7f80u) {                  // something is not finite: the largest of the rest, element by element
    big = 0;
#pragma unroll 1
    for (int c = 0; c < DH / 8; ++c) {
      uint4* v = reinterpret_cast<uint4*>(place + (c >> 3) * 16384 + (((c & 7) ^ (row & 7)) << 4));
      uint4 w = *v;
      big = kv8_max_finite(big, w);
      if (odd) { any |= kv8_zero_non_finite(w); *v = w; }
    }
  }
  ex = kv8_row_exp(big) - lift;
  const float inv = kv8_pow2(-ex);
#pragma unroll 2
  for (int c = 0; c < DH / 8; ++c) {
    uint4* v = reinterpret_cast<uint4*>(place + (c >> 3) * 16384 + (((c & 7) ^ (row & 7)) << 4));
    uint32_t f[4];
    kv8_bf16x8_to_half(*v, inv, f);
    *v = make_uint4(f[0], f[1], f[2], f[3]);
  }
  return any;
}

// The exponent that ku_row_to_operand takes for a row.
template <int DH>
__device__ __forceinline__ int ku_row_exp(const bf16* src, bool on) {
  uint32_t big = 0;
  if (on)
#pragma unroll 4
    for (int c = 0; c < DH / 8; ++c) big = kv8_max_finite(big, *reinterpret_cast<const uint4*>(src + c * 8));
  return kv8_row_exp(big);
}

__device__ __forceinline__ void bulk_prefetch(const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}

constexpr float kKuFits = 65504.f;       // the largest fp16: weights whose sum is at most this fit

// Whether all rows of the warp that exist see new row y (causal).
__device__ __forceinline__ bool ku_all_see(int r, bool on, int rows, int y) { return y < rows && __all_sync(0xffffffffu, !on || y <= r); }

// CHUNK: a prompt's chunk, whose new rows fill key steps that all rows of a tile see; they have a path of their own, which trees and
// few rows do without (it costs the cached steps beside it a sixth: registers).
template <int FMT, int DH, bool CHUNK>
__global__ void __launch_bounds__(kKuThreads, 1) kv8_attn_umma_kernel(const __grid_constant__ Kv8AttnArgs a, const Kv8Plan plan) {
  using Ly = KuLayout<DH>;
  extern __shared__ __align__(1024) uint8_t sm[];
  KuShared& sh = *reinterpret_cast<KuShared*>(sm + Ly::body);
  auto &q_full = sh.q_full, &k_full = sh.k_full, &k_empty = sh.k_empty, &v_full = sh.v_full, &v_empty = sh.v_empty, &sc_full = sh.sc_full;
  auto &c_full = sh.c_full, &c_empty = sh.c_empty;
  auto &s_full = sh.s_full, &p_full = sh.p_full, &pv_done = sh.pv_done;
  auto& s_sc = sh.sc;
  auto& s_bad = sh.bad;
  int& patience = sh.patience;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = blockIdx.x, b = blockIdx.y;
  const Kv8Seq s = kv8_seq(a, b, tid == 0 && h == 0 && blockIdx.z == 0);
  // unit -> (group of row tiles, chunk): chunk-major, so that the full chunks of all sequences start first
  const int groups = plan.paired ? (plan.n_tiles + 1) / 2 : plan.n_tiles;
  // (and the heavier groups: of a chunk the last rows, which see most; else the pairs before a single tile)
  const int nth = (int)blockIdx.z % groups, group = CHUNK ? groups - 1 - nth : nth, chunk_id = (int)blockIdx.z / groups;
  const Kv8Tiles tl = kv8_tiles(a, plan, s, plan.paired ? 2 * group : group);
  pdl_trigger();                   // the join may be scheduled as SMs drain; it waits for this grid
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
  float2(*s_ml)[128] = reinterpret_cast<float2(*)[128]>(sC + 2 * n_slots * Ly::slot);      // (one row tile)

  if (tid == 0) {
    for (int i = 0; i < 2 * kKuSingleSlots; ++i) { mbar_init(&c_full[0][0] + i, 1); mbar_init(&c_empty[0][0] + i, 4); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 4);
      mbar_init(&k_full[i], 4); mbar_init(&k_empty[i], pair ? 2 : 1);      // one release per pipeline that reads the buffer
      mbar_init(&v_full[i], 4); mbar_init(&v_empty[i], pair ? 2 : 1);
      mbar_init(&sc_full[i], 4);
      mbar_init(&sh.drained[i], 1);
      for (int hf = 0; hf < 2; ++hf) { mbar_init(&s_full[i][hf], 1); mbar_init(&p_full[i][hf], 4); mbar_init(&pv_done[i][hf], 1); }
    }
    patience = plan.spin;
    sh.any_bad = 0;
    fence_barrier_init();
  }
  if (tid < kKuBad) s_bad[tid] = 0u;
  if (warp == 2) tmem_alloc(&sh.tmem_base, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;      // pipeline p: columns 256 p + {0, 64}: S of a step's halves, each under its P; 256 p + 128: O

  // pipeline p's i-th step: every step with two row tiles, every other one with a single tile
  auto step_of = [&](int p, int i) { return pair ? i : 2 * i + p; };
  auto steps_of = [&](int p) { return pair ? n : (n + 1 - p) >> 1; };

  if (warp < 4) {
   reg_dec<64>();
   if (warp == 0 || warp == 2) {
    // ---- producers of K and of V: 64 keys a slot, two slots a cached step, a ring each.  A slot's few instructions (a wait,
    // the byte count, a copy per page) take close to a thousand cycles beside the busy softmax warps, so each tensor
    // has a warp of its own, and page ids are read 32 at a time, the next 32 on their way.
    const int is_v = __shfl_sync(0xffffffffu, warp >> 1, 0);
    const int pages = a.c.pt_log2 < 6 ? 64 >> a.c.pt_log2 : 1, bytes = (64 / pages) * DH;      // copies per slot, bytes each
    const int total = is_v || plan.withhold < 0 ? 2 * n_cached : min(2 * n_cached, plan.withhold), col0 = (int)(((long long)j0 << 7) >> a.c.pt_log2), n_cols = (s.len + a.c.pt - 1) >> a.c.pt_log2;
    const size_t page_bytes = (size_t)a.c.hkv * a.c.pt * DH;
    const uint8_t* base = (is_v ? a.c.v : a.c.k) + (size_t)h * a.c.pt * DH;
    uint8_t* ring = sC + is_v * n_slots * Ly::slot;
    uint64_t *const full = c_full[is_v], *const empty = c_empty[is_v];
    auto ids_at = [&](int w) {            // page ids of columns col0 + 32 w + lane
      const int col = col0 + 32 * w + lane;
      return col < n_cols ? kv8_page(a, s.slot, col) : 0;
    };
    int window = 0, ids = ids_at(0), ids_next = ids_at(1), st = 0, use = 0, t = 0;
#pragma unroll 1
    for (; t < total; ++t) {
      const int key = t << 6;             // first key of the slot, from this CTA's first
      const int col = key >> a.c.pt_log2, live = min(pages, (s.len - (j0 << 7) - key + a.c.pt - 1) >> a.c.pt_log2);
      if (col >= 32 * (window + 1)) {
        ++window;
        ids = ids_next;
        ids_next = ids_at(window + 1);
      }
      const int page = __shfl_sync(0xffffffffu, ids, (col + lane) & 31);
      if (use > 0 && !ku_wait(&empty[st], (use - 1) & 1, &patience)) break;
      if (lane == 0) mbar_expect_tx(&full[st], max(live, 0) * bytes);      // 0: the slot lies behind the end, the phase completes
      __syncwarp();
      // two slots are little time for the way from HBM: the lines two steps on are asked into L2
      const int ahead = col + (256 >> a.c.pt_log2);
      const int page4 = __shfl_sync(0xffffffffu, ahead < 32 * (window + 1) ? ids : ids_next, (ahead + lane) & 31);
      if (pair && lane < pages && t + 4 < total) bulk_prefetch(base + page4 * page_bytes + (((t + 4) << 6) & (a.c.pt - 1)) * DH, bytes);
      if (lane < live) bulk_load(ring + st * Ly::slot + lane * bytes, base + page * page_bytes + (key & (a.c.pt - 1)) * DH, bytes, &full[st]);
      if (++st == n_slots) { st = 0; ++use; }
    }
    if (lane == 0) sh.issued[is_v] = make_int2(t, n_slots);
   } else {
    // ---- MMA issuer of pipeline p.  The whole warp runs the loop and one elected lane issues, so descriptors and control
    // flow stay in uniform registers.
    const int p = __shfl_sync(0xffffffffu, warp >> 1, 0);
    const int nh = 2 * steps_of(p);       // half steps of 64 keys
    constexpr uint32_t idesc_s = idesc_f16(128, 64), idesc_o = idesc_f16(128, DH) | kIdescBMnMajor;
    const uint64_t dq = desc_sw128(smem_u32(sQ + (pair ? p : 0) * Ly::tile));
    const uint64_t dk = desc_sw128(smem_u32(sK)), dv = desc_sw128_mn(smem_u32(sV), 16384);
    const uint32_t tS = tmem + p * 256, tO = tS + 128;
    bool ok = nh == 0 || ku_wait(&q_full[pair ? p : 0], 0, &patience);
    // Two things to issue, in whichever order they come ready: S of half step y, once its K is there and P of half y - 2,
    // which lies where it goes, has been used; O += P V of half x, once P is there.  (Waiting for one before the other
    // cost a thousand cycles a half step.)
    int x = 0, y = 0;
#pragma unroll 1
    for (int it = 0; x < nh && ok; ++it) {
      if (y < nh && y <= x + 1) {
        const int j = step_of(p, y >> 1), buf = j & 1, hf = y & 1;
        const bool k_ready = mbar_test_wait(&k_full[buf], (j >> 1) & 1), free = y < 2 || mbar_test_wait(&pv_done[p][hf], ((y >> 1) - 1) & 1);
        if (__all_sync(0xffffffffu, k_ready && free)) {
          tc_fence_after();
          const uint64_t dk1 = dk + (uint32_t)(buf * (Ly::tile >> 4) + hf * (8192 >> 4));
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < DH / 16; ++k) {
              const uint32_t off = ((k >> 2) * 16384 + (k & 3) * 32) >> 4;
              mma_f16(tS + 64 * hf, dq + off, dk1 + off, idesc_s, k > 0 ? 1u : 0u);
            }
            mma_commit(&s_full[p][hf]);
            if (hf == 1) mma_commit(&k_empty[buf]);
          }
          __syncwarp();
          ++y;
          it = 0;
        }
      }
      if (x < y) {
        const int j = step_of(p, x >> 1), buf = j & 1, hf = x & 1;
        const bool p_ready = mbar_test_wait(&p_full[p][hf], (x >> 1) & 1), v_ready = mbar_test_wait(&v_full[buf], (j >> 1) & 1);
        if (__all_sync(0xffffffffu, p_ready && v_ready)) {
          tc_fence_after();
          const uint64_t dv1 = dv + (uint32_t)(buf * (Ly::tile >> 4) + hf * 512);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mma_f16_ts(tO, tS + hf * 64 + k * 8, dv1 + 128 * k, idesc_o, (x > 0 || k > 0) ? 1u : 0u);
            mma_commit(&pv_done[p][hf]);
            if (hf == 1) mma_commit(&v_empty[buf]);
          }
          __syncwarp();
          ++x;
          it = 0;
        }
      }
      if (it > 0) {
        if (__any_sync(0xffffffffu, it > 4 * *(volatile int*)&patience)) { patience = 0; break; }
        __nanosleep(20);
      }
    }
   }
  } else if (warp >= 12) {
    reg_dec<72>();
    // ---- converters: codes (or new rows) to fp16 operand tiles
    // (the first four warps K, the others V and the scales: a key per thread, page id two steps and scales one step ahead)
    const int is_v = (warp - 12) >> 2, ct = (tid - 384) & 127, cw = warp & 3;
    int st = 0, round = 0;           // next code slot and how often the ring has gone round
    const uint8_t* const ring = sC + is_v * n_slots * Ly::slot;
    uint8_t* const tiles = is_v ? sV : sK;
    uint64_t *const full = is_v ? v_full : k_full, *const empty = is_v ? v_empty : k_empty;
    // Eight threads per row, each with 8 codes (an operand chunk) of the row's first 64 and 8 of its second: eight
    // neighbouring threads read 64 bytes in a row and write eight chunks in different banks.  16 rows at a time: one swizzle.
    const int row_in = ct >> 3;
    const uint32_t from = row_in * DH + (ct & 7) * 8, into = row_in * 128 + (((ct & 7) ^ (row_in & 7)) << 4);
    auto publish = [&](uint64_t* bar) {
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    auto page_of = [&](int j) -> int {       // page of this thread's key of step j (the producers report bad ids)
      const int key = ((j0 + j) << 7) + ct;
      if (j >= n_cached || key >= s.len) return -1;
      const int p = a.table[(size_t)s.slot * a.max_pages + (key >> a.c.pt_log2)];
      return (unsigned)p < (unsigned)a.c.n_pages ? p : 0;
    };
    auto scales_of = [&](int page) {
      const size_t ph = (size_t)page * a.c.hkv + h;
      return page < 0 ? make_float2(0.f, 1.f) : make_float2(a.c.ks[ph], a.c.vs[ph]);
    };
    float2 sc = is_v ? scales_of(page_of(0)) : make_float2(0.f, 1.f);
    int page_next = is_v ? page_of(1) : -1;
    bool ok = true;
#pragma unroll 1
    for (int j = 0; j < n && ok; ++j) {
      const int buf = j & 1, use = j >> 1;
      if (use > 0) ok = ku_wait(&empty[buf], (use - 1) & 1, &patience);
      if (!ok) break;
      if (j < n_cached) {
        if (is_v) {
          const float sv = fmaxf(sc.y, kv8_pow2(-100));
          s_sc[buf][ct] = make_float2(sc.x, __log2f(sv));
          __syncwarp();
          if (lane == 0) mbar_arrive(&sc_full[buf]);
          sc = scales_of(page_next);
          page_next = page_of(j + 2);
        }
        const int valid = s.len - ((j0 + j) << 7);        // rows from here on become zero
#pragma unroll 1
        for (int q = 0; q < 2; ++q) {        // 64 keys each
          uint8_t* tile = tiles + buf * Ly::tile + q * 8192;
          ok = ku_wait(&c_full[is_v][st], round & 1, &patience);
          if (!ok) break;
          const uint8_t* src = ring + st * Ly::slot + from;
          uint2 w[4][DH / 64];
#pragma unroll
          for (int it = 0; it < 4; ++it)
#pragma unroll
            for (int c = 0; c < DH / 64; ++c) w[it][c] = *reinterpret_cast<const uint2*>(src + it * 16 * DH + c * 64);
          __syncwarp();
          if (lane == 0) mbar_arrive(&c_empty[is_v][st]);
          if (++st == n_slots) { st = 0; ++round; }
          if (valid < 128) {                 // the end of the cache: code 0 is zero in both formats
#pragma unroll
            for (int it = 0; it < 4; ++it)
              if (q * 64 + row_in + it * 16 >= valid)
#pragma unroll
                for (int c = 0; c < DH / 64; ++c) w[it][c] = make_uint2(0u, 0u);
          }
#pragma unroll
          for (int it = 0; it < 4; ++it)
#pragma unroll
            for (int c = 0; c < DH / 64; ++c) {
              uint4 f;
              kv8_unpack4<FMT>(w[it][c].x, f.x, f.y);
              kv8_unpack4<FMT>(w[it][c].y, f.z, f.w);
              *reinterpret_cast<uint4*>(tile + into + it * 2048 + c * 16384) = f;
            }
        }
        if (!ok) break;
        publish(&full[buf]);
      } else {
        // 128 new rows, one per thread, each divided by a power of two of its own
        const int y0 = (j0 + j - tl.cached) << 7, y = y0 + ct;
        const bool on = y < s.rows;
        const bf16* src = (is_v ? a.v_new : a.k_new) + (size_t)((long long)b * a.rows + (on ? y : 0)) * a.new_stride + (size_t)h * DH;
        int ex;
        const bool odd = ku_row_to_operand<DH>(src, on, tiles + buf * Ly::tile, ct, is_v != 0, is_v ? kv8_lift(FMT) : 0, ex);
        if (is_v) {
          const uint32_t bits = __ballot_sync(0xffffffffu, odd);
          if (lane == 0 && bits != 0u) { s_bad[(y0 >> 5) + cw] = bits; sh.any_bad = 1; }
          // the key's scale is its row's power of two as well: the V group takes it from the row itself
          s_sc[buf][ct] = make_float2(kv8_pow2(ku_row_exp<DH>(a.k_new + (src - a.v_new), on)), (float)ex);
          __syncwarp();
          if (lane == 0) mbar_arrive(&sc_full[buf]);
        }
        publish(&full[buf]);
      }
    }
  } else {
    reg_inc<136>();
    // ---- softmax of pipeline p: thread = row of its tile = tensor-memory lane
    const int p = (warp - 4) >> 2, wq = warp & 3, row = wq * 32 + lane, np = steps_of(p);
    const int tile = tl.first + (pair ? p : 0), i_row = tile * 128 + row;
    const bool on = i_row < Nv;
    const int r = i_row / a.G;            // (of rows that exist)
    const uint32_t tS = tmem + ((uint32_t)(wq * 32) << 16) + p * 256, tO = tS + 128;
    float crow = 0.f;
    if (pair || p == 0) {
      int ex;
      ku_row_to_operand<DH>(a.q + (on ? (size_t)((long long)b * a.rows + r) * a.q_stride + (size_t)(h * a.G + i_row - r * a.G) * DH : 0), on,
                            sQ + (pair ? p : 0) * Ly::tile, row, false, 0, ex);
      crow = a.scale_log2e * kv8_pow2(ex);
      if (!pair) s_ml[0][row].x = crow;
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full[pair ? p : 0]);
    }
    unsigned long long among = 0;         // a tree: the new rows that this row sees, as bits
    if (a.mask != nullptr) {
      const uint8_t* m = a.mask + (size_t)b * a.rows * a.rows;
      const int r_lo = __shfl_sync(0xffffffffu, r, 0), r_hi = min(s.rows - 1, __shfl_sync(0xffffffffu, r, 31));     // the warp's rows
#pragma unroll 4
      for (int x = r_lo; x <= r_hi; ++x) {
        const uint32_t lo = __ballot_sync(0xffffffffu, lane < s.rows && m[x * a.rows + lane] != 0);
        const uint32_t hi = __ballot_sync(0xffffffffu, lane + 32 < s.rows && m[x * a.rows + lane + 32] != 0);
        if (x == r) among = (unsigned long long)hi << 32 | lo;
      }
    }
    if (!pair) {                          // both pipelines of a single tile have the same rows
      asm volatile("bar.sync 1, 256;" ::: "memory");       // the softmax warps
      crow = s_ml[0][row].x;
      asm volatile("bar.sync 1, 256;" ::: "memory");       // s_ml is used again below
    }
    float m_ref = -INFINITY, l = 0.f;
    bool ok = true;
    for (int x = 0; x < 2 * np; ++x) {        // half steps of 64 keys
      const int i = x >> 1, hf = x & 1, j = step_of(p, i), buf = j & 1;
      ok = (hf == 1 || ku_wait(&sc_full[buf], (j >> 1) & 1, &patience)) && ku_wait(&s_full[p][hf], i & 1, &patience);
      if (!ok) break;
      tc_fence_after();
      const float2* scp = &s_sc[buf][hf * 64];
      const bool cached = j < n_cached;
      const int left = s.len - ((j0 + j) << 7);                              // cached keys from this step on
      // a new reference maximum rescales what O holds, once the half step before has been added to it
      auto raise = [&](float mt, float rise) -> bool {
        float alpha = 1.f;
        if (mt > m_ref + rise) {             // also the first visible key (m_ref = -inf)
          alpha = m_ref == -INFINITY ? 1.f : kv8_ex2(m_ref - mt);
          m_ref = mt;
          l *= alpha;
        }
        if (x > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
          if (!ku_wait(&pv_done[p][hf ^ 1], (hf ? i : i - 1) & 1, &patience)) return false;
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
      // New rows in one pass against the reference so far, a scale per key; false: a weight was too large, nothing is written.
      auto new_rows_pass = [&]() -> bool {
        const float mu = m_ref == -INFINITY ? 0.f : m_ref - kKv8Bias;
        float w0 = 0.f, w1 = 0.f;
        uint32_t pk[32];
#pragma unroll
        for (int c0 = 0; c0 < 64; c0 += 16) {
          uint32_t rr[16];
          tmem_ld16(tS + hf * 64 + c0, rr);
          tmem_ld_wait();
#pragma unroll
          for (int q = 0; q < 16; q += 2) {
            const float4 c = *reinterpret_cast<const float4*>(scp + c0 + q);      // two keys
            const float p0 = kv8_ex2(fmaf(__uint_as_float(rr[q]), crow * c.x, c.y - mu));
            const float p1 = kv8_ex2(fmaf(__uint_as_float(rr[q + 1]), crow * c.z, c.w - mu));
            w0 = fmaf(p0, kv8_ex2(-c.y), w0);
            w1 = fmaf(p1, kv8_ex2(-c.w), w1);
            const __half2 v2 = __floats2half2_rn(p0, p1);
            pk[(c0 + q) / 2] = *reinterpret_cast<const uint32_t*>(&v2);
          }
        }
        uint32_t top = 0;                 // of the weights as fp16 bits: 0x7c00 if one was too large
#pragma unroll
        for (int q = 0; q < 32; q += 2) top = __vimax3_u16x2(top, pk[q], pk[q + 1]);
        const bool fine = !on || (max(top & 0xffffu, top >> 16) < 0x7c00u && m_ref != -INFINITY);
        if (__any_sync(0xffffffffu, !fine)) return false;
        l += (w0 + w1) * kKv8Unbias;
        tmem_st32(tS + hf * 64, pk);
        return true;
      };
      if (cached && left >= 128) {
        // 64 cached keys, one set of scales per 16, against the reference so far.  No maximum first: only when a weight does not
        // fit fp16 any more (known from sums of 16, whose limit is a weight 2^7 above the reference or a mean 2^3 above it; and at
        // the very first) the maximum is taken and the half step done again.  The reference then moves whenever the maximum is
        // above it, so that the same weights do not come back to this.
        bool first = x == 0;
#pragma unroll 1
        for (;;) {
          if (first) {
            float mt = -INFINITY;
#pragma unroll 1
            for (int g = 0; g < 4; ++g) {
              uint32_t rr[16];
              tmem_ld16(tS + hf * 64 + g * 16, rr);
              tmem_ld_wait();
              const float2 c = scp[g * 16];
              float x0 = __uint_as_float(rr[0]);
#pragma unroll
              for (int q = 1; q < 15; q += 2) x0 = max3(x0, __uint_as_float(rr[q]), __uint_as_float(rr[q + 1]));
              mt = fmaxf(mt, fmaf(fmaxf(x0, __uint_as_float(rr[15])), crow * c.x, c.y));
            }
            ok = raise(mt, 0.5f);
            if (!ok) break;
          }
          const float mu = m_ref == -INFINITY ? 0.f : m_ref - kKv8Bias;
          float l_new = l, top = 0.f;         // top: the largest sum of 16 weights
          uint32_t pk[32];
          {
            // in phases, not element by element: the compiler keeps the order, and 64 exponentials in a row take a warp 600
            // cycles where the interleaved form took 1000 (the special-function unit's own time is 512)
            float rr[64];
            tmem_ld64(tS + hf * 64, rr);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const float2 c = scp[g * 16];
              const float mul = crow * c.x, sub = c.y - mu;
              const f32x2 mul2 = pack2(mul, mul), sub2 = pack2(sub, sub);
#pragma unroll
              for (int q = 0; q < 16; q += 2)
                unpack2(fma2(pack2(rr[16 * g + q], rr[16 * g + q + 1]), mul2, sub2), rr[16 * g + q], rr[16 * g + q + 1]);
            }
#pragma unroll
            for (int q = 0; q < 64; ++q) rr[q] = kv8_ex2(rr[q]);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              f32x2 ls = pack2(rr[16 * g], rr[16 * g + 1]), lt = pack2(rr[16 * g + 2], rr[16 * g + 3]);
#pragma unroll
              for (int q = 4; q < 16; q += 4) {
                ls = add2(ls, pack2(rr[16 * g + q], rr[16 * g + q + 1]));
                lt = add2(lt, pack2(rr[16 * g + q + 2], rr[16 * g + q + 3]));
              }
              float l0, l1;
              unpack2(add2(ls, lt), l0, l1);
              top = fmaxf(top, l0 + l1);
              l_new = fmaf((l0 + l1) * kKv8Unbias, kv8_ex2(-scp[g * 16].y), l_new);      // back to the weights alone
            }
#pragma unroll
            for (int q = 0; q < 32; ++q) {
              const __half2 v2 = __floats2half2_rn(rr[2 * q], rr[2 * q + 1]);
              pk[q] = *reinterpret_cast<const uint32_t*>(&v2);
            }
          }
          if (first || !__any_sync(0xffffffffu, top > kKuFits)) {
            l = l_new;
            tmem_st32(tS + hf * 64, pk);    // over the scores it came from
            break;
          }
          first = true;
        }
        if (!ok) break;
      } else if (CHUNK && x > 0 && !cached && ku_all_see(r, on, s.rows, ((j0 + j - tl.cached) << 7) + hf * 64 + 63) &&
                 new_rows_pass()) {
        // 64 new rows that every row of the warp sees
      } else {
        // the end of the cache, or new rows that some rows do not see: 16 columns at a time, twice, in little code
        int hi;                           // last visible column, if they are a prefix
        if (cached) hi = left - 1 - hf * 64;
        else hi = min(r, s.rows - 1) - ((j0 + j - tl.cached) << 7) - hf * 64;
        unsigned long long vis = hi < 0 ? 0ull : hi >= 63 ? ~0ull : (2ull << hi) - 1ull;
        if (!cached && a.mask != nullptr) vis = hf == 0 && j0 + j == tl.cached ? among : 0ull;
        if (!on) vis = 0ull;
        float mt = -INFINITY, mu = 0.f;
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {         // the maximum, then the weights
          if (pass == 1) {
            ok = raise(mt, kKv8Rise);
            if (!ok) break;
            mu = m_ref == -INFINITY ? 0.f : m_ref - kKv8Bias;
          }
#pragma unroll 1
          for (int c0 = 0; c0 < 64; c0 += 16) {
            const uint32_t v = (uint32_t)(vis >> c0) & 0xffffu;
            uint32_t pk[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
            if (__any_sync(0xffffffffu, v != 0u)) {    // columns that no row of the warp sees have no weight
              uint32_t rr[16];
              tmem_ld16(tS + hf * 64 + c0, rr);
              tmem_ld_wait();
              float l0 = 0.f, l1 = 0.f;
#pragma unroll
              for (int q = 0; q < 16; ++q) {
                const float2 c = scp[c0 + q];
                float y = fmaf(__uint_as_float(rr[q]), crow * c.x, c.y);
                y = (v >> q) & 1u ? y : -INFINITY;
                if (pass == 0) {
                  mt = fmaxf(mt, y);
                } else {
                  y = kv8_ex2(y - mu);
                  const float w = y * kv8_ex2(-c.y);
                  if (q & 1) l1 += w; else l0 += w;
                  rr[q] = __float_as_uint(y);
                }
              }
              if (pass == 1) {
                l += (l0 + l1) * kKv8Unbias;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                  const __half2 v2 = __floats2half2_rn(__uint_as_float(rr[2 * q]), __uint_as_float(rr[2 * q + 1]));
                  pk[q] = *reinterpret_cast<const uint32_t*>(&v2);
                }
              }
            }
            if (pass == 1) tmem_st8(tS + hf * 64 + c0 / 2, pk);      // over columns read before: c0 / 2 + 7 < c0 + 16
          }
        }
        if (!ok) break;
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[p][hf]);
    }
    if (ok && np > 0) ok = ku_wait(&pv_done[p][1], (np - 1) & 1, &patience);
    if (!pair) {
      s_ml[p][row] = make_float2(m_ref, l);
      tc_fence_before();
      asm volatile("bar.sync 1, 256;" ::: "memory");
    }
    tc_fence_after();
    // ---- results: a pipeline's own tile, or the join of the two pipelines of a single tile (half of the columns each)
    if (__all_sync(0xffffffffu, *(volatile int*)&patience)) {
      const uint32_t tR = tmem + ((uint32_t)(wq * 32) << 16) + 128;
      const bool two = !pair && n > 1;
      const float2 ml0 = pair ? make_float2(m_ref, l) : s_ml[0][row], ml1 = two ? s_ml[1][row] : make_float2(-INFINITY, 0.f);
      const float M = fmaxf(ml0.x, ml1.x);
      float f0 = ml0.y == 0.f ? 0.f : two ? exp2f(ml0.x - M) : 1.f, f1 = ml1.y == 0.f ? 0.f : exp2f(ml1.x - M);
      const float L = ml0.y * f0 + ml1.y * f1;
      const bool whole = tl.split.n == 1;
      if (whole) {                        // finished rows: divided by the sum; without keys, or beyond the rows that exist, zero
        const float inv = L == 0.f || !on ? 0.f : 1.f / L;
        f0 = f0 == 0.f || !on ? 0.f : f0 * inv;
        f1 = f1 == 0.f || !on ? 0.f : f1 * inv;
      }
      const int c_lo = pair ? 0 : p * (DH / 2), c_hi = pair ? DH : c_lo + DH / 2;
      const size_t part = (((size_t)(b * a.c.hkv + h) * plan.n_tiles + tile) * plan.max_chunks + chunk_id) * 128 + row;
      int G = a.G;                        // (opaque: the row's place is worked out again instead of kept in registers through the loop)
      asm volatile("" : "+r"(G));
      const int r_out = i_row / G;
      bf16* out = a.out + ((size_t)((long long)b * a.rows + r_out) * a.hq + h * G + i_row - r_out * G) * DH;
      const bool bad = sh.any_bad != 0 && on;
#pragma unroll 1
      for (int cb = c_lo; cb < c_hi; cb += 8) {
        uint32_t r0[8], r1[8];
        tmem_ld8(tR + (pair ? p * 256 : 0) + cb, r0);
        if (two) tmem_ld8(tR + 256 + cb, r1);
        tmem_ld_wait();
        float o[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          o[q] = f0 == 0.f ? 0.f : __uint_as_float(r0[q]) * kKv8Unbias * f0;
          if (two && f1 != 0.f) o[q] += __uint_as_float(r1[q]) * kKv8Unbias * f1;
        }
        if (bad) {                        // values that are not finite reach exactly the rows that see them
#pragma unroll 1
          for (int y = 0; y < s.rows; ++y) {
            if (!((s_bad[y >> 5] >> (y & 31)) & 1u) || !kv8_sees(a, b, r_out, y)) continue;
            const uint4 v = *reinterpret_cast<const uint4*>(a.v_new + (size_t)((long long)b * a.rows + y) * a.new_stride + (size_t)h * DH + cb);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const float z = __uint_as_float(q & 1 ? w[q / 2] & 0xffff0000u : w[q / 2] << 16);
              if (!isfinite(z)) o[q] += z;
            }
          }
        }
        if (i_row < N) {
          if (whole) {
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const __nv_bfloat162 v2 = __floats2bfloat162_rn(o[2 * q], o[2 * q + 1]);
              w[q] = *reinterpret_cast<const uint32_t*>(&v2);
            }
            DART_CHECK(r_out < a.rows && cb < DH, a.status)
            *reinterpret_cast<uint4*>(out + cb) = make_uint4(w[0], w[1], w[2], w[3]);
          } else {
            float4* dst = reinterpret_cast<float4*>(plan.o_part + part * DH + cb);
            DART_CHECK(tile < plan.n_tiles && chunk_id < plan.max_chunks, a.status) {
              dst[0] = make_float4(o[0], o[1], o[2], o[3]);
              dst[1] = make_float4(o[4], o[5], o[6], o[7]);
            }
          }
        }
        __syncwarp();
      }
      if (!whole && c_lo == 0 && i_row < N) *reinterpret_cast<float2*>(plan.ml_part + part * 2) = make_float2(M, L);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (patience == 0) {             // a wait ran out: leave no copy and no MMA in flight behind
    tc_fence_after();
    if (warp == 0 || warp == 2) {
      const int2 last = sh.issued[warp >> 1];
#pragma unroll 1
      for (int u = max(0, last.x - last.y); u < last.x; ++u)
#pragma unroll 1
        for (int it = 0; it < 1000000 && !mbar_test_wait(&c_full[warp >> 1][u % last.y], (u / last.y) & 1); ++it) {}
    } else if (warp == 1 || warp == 3) {
      if (elect_one()) mma_commit(&sh.drained[warp >> 1]);
      __syncwarp();
#pragma unroll 1
      for (int it = 0; it < 1000000 && !mbar_test_wait(&sh.drained[warp >> 1], 0); ++it) {}
    }
    if (tid == 0) kv8_report(a.status, DEV_TIMEOUT);
    tc_fence_before();
    __syncthreads();
  }
  if (warp == 2) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

// Key steps of a CTA.  A CTA's start and end (queries, the first copies, the first scores, its result) cost as much as five or
// six steps, and a partial result is written, read again and joined, so the keys are split only as far as one wave of
// CTAs, one to an SM, goes.  (Measured, steps per CTA: 16 ragged sequences of up to 65 steps, 256 cells: 65 steps 175 us, 33: 203,
// 16: 238; prompt chunk, 256 cells of 44: 44 steps 247 us, 22: 316; one tree in pairs, 16 cells of 33 steps: 4 steps 32.4 us, 3: 35.5, 8:
// 37.6.)  By max_len, not by the lengths: one tree over 4096 keys 27 us with that bound, 65 with 32768, 97 with 131072.
// A step of two row tiles takes about 2.2 us and the CTA around it 15; a step of one tile 1.6 us and its CTA 11: two tiles
// are cheaper by the row, one tile is done sooner where the GPU is not full anyway (one tree over 33 steps,
// 3 tiles of 8 heads: 27.0 us in single tiles, 32.4 in pairs).
void kv8_umma_plan(const Kv8AttnArgs& a, Kv8Plan& p) {
  constexpr int kSms = 148, kMinSteps = 4;
  p.n_tiles = (a.rows * a.G + 127) / 128;
  const long long heads = (long long)a.batch * a.c.hkv;
  const int steps = (int)(((long long)a.max_len + 127) / 128) + (a.k_new != nullptr ? (a.rows + 127) / 128 : 0);
  const long long all = ((long long)a.max_len + 127) / 128 + (a.rows + 127) / 128;       // whether or not there are new rows
  double best = 0.0;
  long long most = 0;             // parts that no smaller max_len exceeds, in either form
  for (int paired = 0; paired < 2; ++paired) {
    if (paired && p.n_tiles == 1) break;
    const long long groups = paired ? (p.n_tiles + 1) / 2 : p.n_tiles, cells = groups * heads;
    const long long parts = cells >= kSms ? 1 : kSms / cells;
    long long chunk = (steps + parts - 1) / parts;
    if (chunk < kMinSteps) chunk = kMinSteps;
    const long long longest = all * groups / 63487 + 1;                                   // the grid's third dimension
    if (chunk < longest) chunk = longest;
    const double waves = cells >= kSms ? (double)cells / kSms : 1.0, cost = waves * (paired ? 15.0 + 2.2 * chunk : 11.0 + 1.6 * chunk);
    if (paired == 0 || cost < best) {
      best = cost;
      p.paired = paired;
      p.chunk = (int)chunk;
    }
    if (parts > most) most = parts;
  }
  p.max_chunks = kv8_split(steps, p.chunk, 1).n;
  if (most > (all + kMinSteps - 1) / kMinSteps) most = (all + kMinSteps - 1) / kMinSteps;
  p.bytes = most > 1 ? (size_t)heads * p.n_tiles * 128 * (size_t)most : 0;                // partial rows
}

namespace {
template <int FMT, int DH, bool CHUNK>
cudaError_t launch_kernel(const Kv8AttnArgs& a, const Kv8Plan& p, cudaStream_t st) {
  const auto kernel = kv8_attn_umma_kernel<FMT, DH, CHUNK>;
  const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), KuLayout<DH>::smem);
  if (e != cudaSuccess) return e;
  kernel<<<dim3(a.c.hkv, a.batch, (p.paired ? (p.n_tiles + 1) / 2 : p.n_tiles) * p.max_chunks), kKuThreads, KuLayout<DH>::smem, st>>>(a, p);
  return cudaGetLastError();
}
template <int FMT, int DH>
cudaError_t launch(const Kv8AttnArgs& a, const Kv8Plan& p, cudaStream_t st) {
  return a.mask == nullptr && a.k_new != nullptr && a.rows > 128 ? launch_kernel<FMT, DH, true>(a, p, st) : launch_kernel<FMT, DH, false>(a, p, st);
}
}  // namespace

cudaError_t launch_kv8_attn_umma(const Kv8AttnArgs& a, const Kv8Plan& p, cudaStream_t st) {
  if (a.c.format == KV8_E4M3) return a.c.dh == 128 ? launch<KV8_E4M3, 128>(a, p, st) : launch<KV8_E4M3, 64>(a, p, st);
  return a.c.dh == 128 ? launch<KV8_INT8, 128>(a, p, st) : launch<KV8_INT8, 64>(a, p, st);
}

}  // namespace dart
