// Pages of the 8-bit cache: fork, reserve with copy-on-write, release, compact.
//
// The one truth about a page is its reference count (0: free); there is no free list to keep consistent.  Pages are
// handed out lowest id first, in list order, so that two runs of the same calls give the same tables.  Reserve and
// compact are a planning kernel of one block (prefix sums over the counts; a few microseconds) that leaves a list of
// (source, destination) pages in the workspace, and a copy kernel over the list, whose length only the device knows.  The
// copies run at memory speed (48 pages of 16 layers, 200 MB read and written: 27 us); what the small kernels before them
// cost is their launches and chains of dependent reads, so every kernel here is launched ahead of its predecessor's end
// (pdl_wait) and the planning kernels compare lists in shared memory.  Measured (device time, back to back in a CUDA
// graph; through Python 44, 18 and 146), with the restoring of the tables between two passes (2 us): 16 sequences forked three
// times, then all 64 reserved, 40.8 us; one fork and reserve of a
// short sequence 9.8 us; compaction after releasing half of 64 sequences (169 pages of 16 layers, 709 MB) 137 us, the
// copies alone 122 = 0.89 of the copy peak.
#include "kv8.cuh"

namespace dart {

constexpr int kPgThreads = 1024;
// Workspace, in ints: [0] entries of the copy list; [16..]: destinations, sources (-1: nothing to copy), slots, columns;
// compact uses the third array for the new ids.
constexpr int kPgHead = 16;
size_t kv8_pages_workspace(int n_pages) { return ((size_t)kPgHead + 4 * (size_t)n_pages) * sizeof(int); }

// Exclusive prefix sum of v <= 2^24 + 1 over the block's threads; *total gets the sum.  sh: 33 ints; the caller syncs before
// reuse.  A warp's sum counts as 2^25 at most, so that nothing overflows: sums above 2^24 are above it, no more.
__device__ __forceinline__ int block_scan(int v, int* sh, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) sh[warp] = min(x, 1 << 25);
  __syncthreads();
  if (warp == 0) {
    const int s = lane < (int)(blockDim.x >> 5) ? sh[lane] : 0;
    int t = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) t += y;
    }
    sh[lane] = t - s;
    if (lane == 31) sh[32] = t;
  }
  __syncthreads();
  *total = sh[32];
  return sh[warp] + x - v;
}

// How many of the first n entries of a 16-byte aligned list in shared memory equal x.
__device__ __forceinline__ int count_before(const int* list, int n, int x) {
  int c = 0, t = 0;
#pragma unroll 4
  for (; t + 4 <= n; t += 4) {
    const int4 v = *reinterpret_cast<const int4*>(list + t);
    c += (v.x == x) + (v.y == x) + (v.z == x) + (v.w == x);
  }
  for (; t < n; ++t) c += list[t] == x;
  return c;
}

__global__ void __launch_bounds__(256) kv8_fork_kernel(const Kv8PagesArgs p, const int* src, const int* dst, int n, int* status) {
  const int i = blockIdx.x, tid = threadIdx.x;
  pdl_wait();
  pdl_trigger();
  const int s = src[i], d = dst[i];
  int bad = s < 0 || s >= p.max_seqs || d < 0 || d >= p.max_seqs || s == d;
  for (int t = tid; t < n; t += blockDim.x) bad |= dst[t] == s || (t < i && dst[t] == d);
  int len = 0;
  if (!bad) {      // slot s is nobody's destination, so no block of this call writes it
    len = p.seq_lens[s];
    bad = len < 0 || (long long)len > (long long)p.max_pages * p.pt || p.seq_lens[d] != 0;
    for (int j = tid; j < p.max_pages; j += blockDim.x) bad |= p.table[(size_t)d * p.max_pages + j] != -1;
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) kv8_report(status, KV8_BAD_ARG);
    return;
  }
  const int cols = (len + p.pt - 1) / p.pt;
  for (int j = tid; j < cols; j += blockDim.x) {
    const int e = p.table[(size_t)s * p.max_pages + j];
    if (e != kKv8GivenBack && (e < 0 || e >= p.n_pages)) { kv8_report(status, KV8_BAD_ARG); continue; }
    DART_CHECK(d < p.max_seqs && j < p.max_pages, status) {
      p.table[(size_t)d * p.max_pages + j] = e;
      if (e >= 0) atomicAdd(&p.ref[e], 1);
    }
  }
  if (tid == 0) p.seq_lens[d] = len;
}

__global__ void __launch_bounds__(256) kv8_release_kernel(const Kv8PagesArgs p, const int* seqs, int* status) {
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x, tid = threadIdx.x, s = seqs[i];
  int bad = s < 0 || s >= p.max_seqs;
  for (int t = tid; t < i; t += blockDim.x) bad |= seqs[t] == s;
  if (__syncthreads_or(bad)) {
    if (tid == 0) kv8_report(status, KV8_BAD_ARG);
    return;
  }
  for (int j = tid; j < p.max_pages; j += blockDim.x) {
    int* e = p.table + (size_t)s * p.max_pages + j;
    const int page = *e;
    if (page == -1) continue;
    *e = -1;
    if (page == kKv8GivenBack) continue;
    if (page < 0 || page >= p.n_pages) { kv8_report(status, KV8_BAD_ARG); continue; }
    if (atomicSub(&p.ref[page], 1) <= 0) { atomicAdd(&p.ref[page], 1); kv8_report(status, KV8_BAD_ARG); }
  }
  if (tid == 0) p.seq_lens[s] = 0;
}

// Columns [sinks / pt rounded up, (len - window + 1) / pt) lie behind the window of every row to come and hold no sink.  A block takes
// kTrimCols columns of a slot at a time.  What bounds it is a launch and a chain of dependent reads (slot, length, entry, count), so the
// entries of a thread are read together: 64 slots with 250000 entries 26.5 us with one block to a slot and one entry after the other, 7.3 so
// (2 of them the restoring of the tables between two calls).
constexpr int kTrimEach = 4, kTrimCols = 256 * kTrimEach;
__global__ void __launch_bounds__(256) kv8_trim_kernel(const Kv8PagesArgs p, const int* seqs, int window, int sinks, int* status) {
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x, tid = threadIdx.x, s = seqs[i];
  int bad = s < 0 || s >= p.max_seqs;
  const int len = bad ? 0 : p.seq_lens[s];
  for (int t = tid; t < i; t += blockDim.x) bad |= seqs[t] == s;
  bad |= len < 0 || (long long)len > (long long)p.max_pages * p.pt;
  if (__syncthreads_or(bad)) {
    if (tid == 0 && blockIdx.y == 0) kv8_report(status, KV8_BAD_ARG);
    return;
  }
  const int end = len >= window ? (len - window + 1) / p.pt : 0, begin = sinks / p.pt + (sinks % p.pt != 0);
  int* row = p.table + (size_t)s * p.max_pages;
#pragma unroll 1
  for (int j0 = begin + blockIdx.y * kTrimCols; j0 < end; j0 += gridDim.y * kTrimCols) {
    int page[kTrimEach];
#pragma unroll
    for (int q = 0; q < kTrimEach; ++q) {
      const int j = j0 + q * 256 + tid;
      page[q] = j < end ? row[j] : kKv8GivenBack;
    }
#pragma unroll
    for (int q = 0; q < kTrimEach; ++q) {
      if (page[q] == kKv8GivenBack) continue;
      if (page[q] < 0 || page[q] >= p.n_pages) { kv8_report(status, KV8_BAD_ARG); continue; }
      const int j = j0 + q * 256 + tid;
      DART_CHECK(s < p.max_seqs && j < p.max_pages, status) row[j] = kKv8GivenBack;
      if (atomicSub(&p.ref[page[q]], 1) <= 0) { atomicAdd(&p.ref[page[q]], 1); kv8_report(status, KV8_BAD_ARG); }
    }
  }
}

__global__ void __launch_bounds__(kPgThreads) kv8_reserve_plan_kernel(const Kv8PagesArgs p, const int* seqs, const int* n_new, int n, int* ws,
                                                                      int* status) {
  __shared__ int sh[33], s_lo[kPgThreads], s_start[kPgThreads + 1];
  __shared__ __align__(16) int s_slot[kPgThreads], s_shared[kPgThreads];
  const int tid = threadIdx.x;
  pdl_wait();
  pdl_trigger();
  int* dst = ws + kPgHead;
  int *src = dst + p.n_pages, *slot = src + p.n_pages, *column = slot + p.n_pages;
  // the columns [lo, lo + width) that item tid wants to write
  const int m = tid < n ? n_new[tid] : 0;
  s_slot[tid] = m != 0 ? seqs[tid] : -1;         // an entry without positions claims no slot
  __syncthreads();
  int width = 0, lo = 0;
  if (tid < n) {
    const int s = m != 0 ? s_slot[tid] : seqs[tid];
    bool bad = s < 0 || s >= p.max_seqs || m < 0;
    bad |= m != 0 && count_before(s_slot, tid, s) > 0;
    const int len = bad ? 0 : p.seq_lens[s];
    if (len < 0 || (!bad && (long long)len + m > (long long)p.max_pages * p.pt)) bad = true;
    if (bad) kv8_report(status, KV8_BAD_ARG);
    else if (m > 0) { lo = len / p.pt; width = (len + m - 1) / p.pt + 1 - lo; }
  }
  s_lo[tid] = lo;
  int total_cols, total_need = 0;
  const int start = block_scan(min(width, p.n_pages + 1), sh, &total_cols);
  // every listed column ends up with a page of its own: more columns than pages cannot be had
  const bool too_many = total_cols > p.n_pages;
  if (too_many) total_cols = 0;
  s_start[tid] = start;
  if (tid == 0) s_start[kPgThreads] = total_cols;
  __syncthreads();
  // (item, column) pairs in list order: which need a page
  for (int base = 0; base < total_cols; base += kPgThreads) {
    const int f = base + tid;
    int need = 0, old = -1, s = 0, j = 0, shared = -1, refs = 0, a = 0;
    if (f < total_cols) {
      int b = kPgThreads - 1;                    // the last item that starts at or before f
      while (a < b) {
        const int c = (a + b + 1) >> 1;
        if (s_start[c] <= f) a = c; else b = c - 1;
      }
      s = s_slot[a];
      j = s_lo[a] + f - s_start[a];
      const int e = p.table[(size_t)s * p.max_pages + j];
      if (e == -1) need = 1;
      else if (e < 0 || e >= p.n_pages) kv8_report(status, KV8_BAD_ARG);
      else if ((refs = p.ref[e]) > 1) shared = e;
    }
    // a shared page: earlier sharers of the list copy first, the last one keeps it.  (A page sits in the same column of all
    // its sharers, so a pair further up the list with the same page is another sharer.)
    if (__syncthreads_or(shared >= 0)) {
      s_shared[tid] = shared;
      __syncthreads();
      if (shared >= 0) {
        int rank = count_before(s_shared, tid, shared);
        for (int t = 0; base > 0 && t < a; ++t) {          // sharers in earlier rounds of a list of more than 1024 pairs
          const int width_t = s_start[t + 1] - s_start[t];
          if (j >= s_lo[t] && j < s_lo[t] + width_t && s_start[t] + j - s_lo[t] < base)
            rank += p.table[(size_t)s_slot[t] * p.max_pages + j] == shared;
        }
        if (rank < refs - 1) { need = 1; old = shared; }
      }
    }
    int here;
    const int k = total_need + block_scan(need, sh, &here);
    DART_CHECK(!need || (k >= 0 && k < p.n_pages), status)
    if (need) { src[k] = old; slot[k] = s; column[k] = j; }
    total_need += here;
  }
  __syncthreads();
  // the lowest free pages
  int found = 0;
  for (int base = 0; base < p.n_pages && found < total_need; base += 4 * kPgThreads) {
    int free_bits = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int id = base + tid * 4 + q;
      if (id < p.n_pages && p.ref[id] == 0) free_bits |= 1 << q;
    }
    int here;
    int k = found + block_scan(__popc(free_bits), sh, &here);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if ((free_bits >> q) & 1) {
        if (k < total_need) dst[k] = base + tid * 4 + q;
        ++k;
      }
    found += here;
  }
  __syncthreads();
  const bool ok = !too_many && found >= total_need;
  if (ok)
    for (int k = tid; k < total_need; k += kPgThreads) {
      const int page = dst[k];
      DART_CHECK(page >= 0 && page < p.n_pages && slot[k] >= 0 && slot[k] < p.max_seqs && column[k] >= 0 && column[k] < p.max_pages && src[k] < p.n_pages, status) {
        p.table[(size_t)slot[k] * p.max_pages + column[k]] = page;
        p.ref[page] = 1;
        if (src[k] >= 0) atomicSub(&p.ref[src[k]], 1);
      }
    }
  if (tid == 0) {
    ws[0] = ok ? total_need : 0;
    if (!ok) kv8_report(status, KV8_CAPACITY);
  }
}

__global__ void __launch_bounds__(kPgThreads) kv8_compact_plan_kernel(const Kv8PagesArgs p, int* ws, int* n_live_out, int* status) {
  __shared__ int sh[33];
  const int tid = threadIdx.x;
  pdl_wait();
  pdl_trigger();
  int* dst = ws + kPgHead;
  int *src = dst + p.n_pages, *to = src + p.n_pages;
  int mine = 0, n_live;
  for (int id = tid; id < p.n_pages; id += kPgThreads) mine += p.ref[id] > 0;
  block_scan(mine, sh, &n_live);
  int n_src = 0, n_dst = 0;      // as many live pages at n_live and above as free ones below it
  for (int base = 0; base < p.n_pages; base += 4 * kPgThreads) {
    int moves = 0, holes = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int id = base + tid * 4 + q;
      if (id >= p.n_pages) continue;
      to[id] = id;
      const bool live = p.ref[id] > 0;
      if (live && id >= n_live) moves |= 1 << q;
      if (!live && id < n_live) holes |= 1 << q;
    }
    int here_src, here_dst;
    int ks = n_src + block_scan(__popc(moves), sh, &here_src), kd = n_dst + block_scan(__popc(holes), sh, &here_dst);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int id = base + tid * 4 + q;
      DART_CHECK(ks < p.n_pages && kd < p.n_pages, status) {
        if ((moves >> q) & 1) src[ks++] = id;
        if ((holes >> q) & 1) dst[kd++] = id;
      }
    }
    n_src += here_src;
    n_dst += here_dst;
  }
  __syncthreads();
  for (int k = tid; k < n_src; k += kPgThreads) {
    const int s = src[k], d = dst[k];
    to[s] = d;
    p.ref[d] = p.ref[s];
    p.ref[s] = 0;
  }
  if (tid == 0) {
    ws[0] = n_src;
    if (n_live_out != nullptr) *n_live_out = n_live;
  }
}

// Copies the listed pages of every layer, and (compact) renames the table's entries.
constexpr int kCpThreads = 256, kCpChunk = kCpThreads * 64;   // bytes a block copies at a time
__global__ void __launch_bounds__(kCpThreads) kv8_copy_pages_kernel(const Kv8PagesArgs p, const Kv8PoolArgs c, const int* ws, int rename,
                                                                     int* status) {
  pdl_wait();
  const int tid = threadIdx.x, count = ws[0];
  const int* dst = ws + kPgHead;
  const int *src = dst + p.n_pages, *to = src + p.n_pages;
  if (rename) {
    const long long cells = (long long)p.max_seqs * p.max_pages;
    for (long long i = (long long)blockIdx.x * kCpThreads + tid; i < cells; i += (long long)gridDim.x * kCpThreads) {
      const int e = p.table[i];
      if (e >= 0 && e < p.n_pages && to[e] != e) p.table[i] = to[e];
    }
  }
  const int parts = (int)((c.slab + kCpChunk - 1) / kCpChunk);
  const long long units = (long long)count * c.n_layers * 2 * parts;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    long long x = u;
    const int part = (int)(x % parts); x /= parts;
    const int is_v = (int)(x & 1); x >>= 1;
    const int layer = (int)(x % c.n_layers), k = (int)(x / c.n_layers);
    const int s = src[k], d = dst[k];
    if (s < 0) continue;
    const size_t sp = (size_t)layer * c.n_pages + s, dp = (size_t)layer * c.n_pages + d;
    uint8_t* pool = is_v ? c.v : c.k;
    const uint4* from = reinterpret_cast<const uint4*>(pool + sp * c.slab);
    uint4* into = reinterpret_cast<uint4*>(pool + dp * c.slab);
    const int n16 = (int)(c.slab / 16), at = part * (kCpChunk / 16) + tid;
    uint4 v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (at + q * kCpThreads < n16) v[q] = from[at + q * kCpThreads];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (at + q * kCpThreads < n16) {
        DART_CHECK(d >= 0 && d < p.n_pages && layer < c.n_layers, status)
        into[at + q * kCpThreads] = v[q];
      }
    if (part == 0) {
      float* sc = is_v ? c.vs : c.ks;
      for (int h = tid; h < c.hkv; h += kCpThreads) {
        DART_CHECK(d >= 0 && d < p.n_pages, status)
        sc[dp * c.hkv + h] = sc[sp * c.hkv + h];
      }
    }
  }
}

namespace {
constexpr int kCpGrid = 148 * 8;
}  // namespace

cudaError_t launch_kv8_fork(const Kv8PagesArgs& p, const int* src, const int* dst, int n, int* status, cudaStream_t st) {
  return launch_ahead(kv8_fork_kernel, dim3(n), 256, 0, st, p, src, dst, n, status);
}

cudaError_t launch_kv8_release(const Kv8PagesArgs& p, const int* seqs, int n, int* status, cudaStream_t st) {
  return launch_ahead(kv8_release_kernel, dim3(n), 256, 0, st, p, seqs, status);
}

cudaError_t launch_kv8_trim(const Kv8PagesArgs& p, const int* seqs, int n, int window, int sinks, int* status, cudaStream_t st) {
  const int blocks = (p.max_pages + kTrimCols - 1) / kTrimCols;
  return launch_ahead(kv8_trim_kernel, dim3(n, blocks < 16 ? blocks : 16), 256, 0, st, p, seqs, window, sinks, status);
}

cudaError_t launch_kv8_reserve(const Kv8PagesArgs& p, const Kv8PoolArgs& c, const int* seqs, const int* n_new, int n, int* ws, int* status,
                               cudaStream_t st) {
  const cudaError_t e = launch_ahead(kv8_reserve_plan_kernel, dim3(1), kPgThreads, 0, st, p, seqs, n_new, n, ws, status);
  if (e != cudaSuccess) return e;
  return launch_ahead(kv8_copy_pages_kernel, dim3(kCpGrid), kCpThreads, 0, st, p, c, ws, 0, status);
}

cudaError_t launch_kv8_compact(const Kv8PagesArgs& p, const Kv8PoolArgs& c, int* n_live, int* ws, int* status, cudaStream_t st) {
  const cudaError_t e = launch_ahead(kv8_compact_plan_kernel, dim3(1), kPgThreads, 0, st, p, ws, n_live, status);
  if (e != cudaSuccess) return e;
  return launch_ahead(kv8_copy_pages_kernel, dim3(kCpGrid), kCpThreads, 0, st, p, c, ws, 1, status);
}

}  // namespace dart
