// Pages of a cache handed on: the accepted tokens of a drafted tree, sequences that go on from others, copies of pages.
#include "common.h"
#include "launch.h"
#include "paged.h"

namespace blossom {
namespace paged {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int page_of(const Args &a, const int *table, int pos)
{
  if (pos < 0 || pos >= a.cap) return -1;
  const int id = table[pos >> a.page_shift];
  return id >= 0 && id < a.n_pages ? id : -1;
}

}  // namespace

// Rows past + keep[i] move to past + i, i ascending.  A thread owns 16 bytes of every row (of K or of V, of one key/value head), so what it
// reads later never lies where it wrote: keep[j] >= j > i for j > i.  No thread waits for another.
__global__ __launch_bounds__(kThreads) void accept_kernel(Args a, Accept x, int row_chunks)
{
  constexpr int AHEAD = 8;
  const int lane = threadIdx.x & 63;
  const int per = 2 * a.G * row_chunks, groups = (per + kThreads - 1) / kThreads;  // threads and workgroups of a sequence
  const int s = blockIdx.x / groups, at = (blockIdx.x - s * groups) * kThreads + threadIdx.x;
  const int first = token_at(a, s), n = max(token_at(a, s + 1) - first, 0);
  const int raw = a.kv_len[s], past = max(raw, 0) - n;
  const int *keep = x.keep + (size_t)s * x.width;
  const int *table = a.page_table + s * a.table_seq;
  // how many are kept: a lane an entry
  int kept = 0;
  for (int i0 = 0; i0 < x.width; i0 += 64) {
    const int i = i0 + lane;
    const int mine = i < x.width ? keep[i] : -1, before = i == 0 || i >= x.width ? -1 : keep[i - 1];
    const unsigned long long good = __ballot(mine > before && mine < n && mine >= 0);
    const int run = good == ~0ull ? 64 : __builtin_ctzll(~good);
    kept += run;
    if (run < 64) break;
  }
  if (at == 0 && x.new_len) x.new_len[s] = past + kept;
  if (at >= per) return;
  const int chunk = at % row_chunks, head = at / row_chunks;  // K's heads, then V's
  uint4 *cache = reinterpret_cast<uint4 *>(head < a.G ? a.K_cache : a.V_cache);
  const int g = head < a.G ? head : head - a.G, page = 1 << a.page_shift;
  auto cell = [&](int id, int pos) __attribute__((always_inline)) {
    return cache + (((size_t)id * a.G + g) * page + (pos & (page - 1))) * row_chunks + chunk;
  };
  for (int i0 = 0; i0 < kept; i0 += AHEAD) {
    uint4 v[AHEAD];
    uint4 *to[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      to[k] = nullptr;
      const int i = i0 + k;
      if (i >= kept || keep[i] == i) continue;
      const int src = page_of(a, table, past + keep[i]), dst = page_of(a, table, past + i);
      if (src < 0 || dst < 0) continue;
      v[k] = *cell(src, past + keep[i]);
      to[k] = cell(dst, past + i);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (to[k]) *to[k] = v[k];
  }
}

bool launch_accept(const Args &a, const Accept &x, hipStream_t st)
{
  const int row_chunks = a.d * (a.dtype == 0 ? 4 : 2) / 16;
  const long blocks = (long)a.S * ((2l * a.G * row_chunks + kThreads - 1) / kThreads);
  if (!countable(blocks, kThreads)) return false;
  hipLaunchKernelGGL(accept_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, st, a, x, row_chunks);
  return true;
}

// ---- fork ----
//
// Sequence n goes on from parent q with L = len[q] positions, of which `full` pages are whole.  Whole pages are shared.  Of the pages from
// there on, up to those that L + grow positions need, the eldest of q's children keeps what nobody else holds; all others are fresh, the
// one with the last L mod page rows a copy.  refs' = refs - entries of the old table + entries of the new one; fresh pages are those that
// nobody holds then and no copy reads, the lowest first, to the sequences in order.

// Sequences take a wavefront each, fresh pages one workgroup: two launches between which the counts settle.  A launch takes longer than its
// work: a fork of 512 sequences of up to 4040 positions takes four launches of 4 to 9 us, mostly chains of loads from one to the next.
//
// What a new sequence takes over.
struct Heir {
  int q, len, full, part, need;  // (q < 0: nothing)
  __device__ __forceinline__ Heir(const Args &a, const Fork &x, int n)
  {
    q = x.parent[n];
    if (q < 0 || q >= a.S) q = -1;
    len = q < 0 ? 0 : min(max(a.kv_len[q], 0), a.cap);
    full = len >> a.page_shift;
    part = len & ((1 << a.page_shift) - 1);
    need = q < 0 ? 0 : (int)((min((long)len + x.grow, (long)a.cap) + (1 << a.page_shift) - 1) >> a.page_shift);
  }
};
__device__ __forceinline__ int valid(const Args &a, int id) { return id >= 0 && id < a.n_pages ? id : -1; }

// ---- by a wavefront: new sequence n, and what becomes of old sequence n ----

// Its row of the new table, fresh pages as -2, -3, .. in order, how many those are, and which page it copies.
__device__ __forceinline__ void fork_row(const Args &a, const Fork &x, int n, int lane)
{
  const Heir h(a, x, n);
  bool elder = false;  // does an earlier one go on from the same parent?
  for (int i = lane; i < n; i += 64) elder = elder || x.parent[i] == h.q;
  const bool eldest = h.q >= 0 && !__any(elder);
  const int *from = a.page_table + (size_t)max(h.q, 0) * a.max_pages;
  int *to = x.table + (size_t)n * a.max_pages;
  int fresh = 0, copy = -1;
  for (int i0 = 0; i0 < a.max_pages; i0 += 64) {
    const int i = i0 + lane;
    const int old = i < h.need ? valid(a, from[i]) : -1;
    const bool taken = i < h.full || (i < h.need && eldest && old >= 0 && x.refs[old] == 1), asks = i < h.need && !taken;
    const unsigned long long all = __ballot(asks);
    const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(all >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)all, 0));
    if (asks && i == h.full && h.part > 0) copy = old;
    if (i < a.max_pages) to[i] = taken ? old : asks ? -2 - (fresh + before) : -1;
    fresh += __builtin_popcountll(all);
  }
  const unsigned long long copies = __ballot(copy >= 0);
  copy = __builtin_amdgcn_readlane(copy, copies ? __builtin_ctzll(copies) : 0);
  if (lane == 0) {
    x.fresh[n] = fresh;
    x.len[n] = h.len;
    x.at[n] = make_int2(h.full, eldest);
    x.copies[3 * n] = copy;
    x.copies[3 * n + 2] = h.part;
  }
}
// Who holds a page then: one more for every page that a younger one shares, one less for those that neither the eldest takes over.
__device__ __forceinline__ void fork_refs(const Args &a, const Fork &x, int n, int lane)
{
  if (n < x.N) {
    const int2 at = x.at[n];
    const int copy = x.copies[3 * n];
    const int *row = x.table + (size_t)n * a.max_pages;
    for (int i = lane; i < (at.y ? 0 : at.x); i += 64)
      if (row[i] >= 0) atomicAdd(x.new_refs + row[i], 1);
    if (lane == 0 && copy >= 0) atomicAdd(x.held + copy, 1);
  }
  if (n >= a.S) return;
  int heir = x.N;
  for (int i = lane; i < x.N; i += 64)
    if (x.parent[i] == n) heir = min(heir, i);
  heir = x.N - wave_max(x.N - heir);  // the eldest
  const int *from = a.page_table + (size_t)n * a.max_pages;
  const int *row = x.table + (size_t)min(heir, x.N - 1) * a.max_pages;
  for (int i = lane; i < a.max_pages; i += 64) {
    const int old = valid(a, from[i]), now = heir == x.N ? -1 : row[i];
    if (old >= 0 && now != old) atomicSub(x.new_refs + old, 1);
  }
}

// Fresh pages, by one workgroup of 1024.
__device__ __forceinline__ void fork_give(const Args &a, const Fork &x, int tid)
{
  constexpr int AT_ONCE = 4, NEAR = 4096;
  __shared__ int sums[16], begin_s[NEAR];
  const int lane = tid & 63, wv = tid >> 6;
  // exclusive sums over the workgroup; *total: of all
  auto scan = [&](int v, int *total) -> int {
    const int upto = wave_scan(v);
    __syncthreads();
    if (lane == 63) sums[wv] = upto;
    __syncthreads();
    const int s = lane < 16 ? sums[lane] : 0, t = wave_scan(s);
    *total = __builtin_amdgcn_readlane(t, 15);
    return __shfl(t - s, wv) + upto - v;
  };
  auto look = [&](int p0) -> unsigned {
    unsigned free = 0;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int p = p0 + tid * AT_ONCE + i;
      if (p < a.n_pages && x.new_refs[p] == 0 && x.held[p] == 0) free |= 1u << i;
    }
    return free;
  };
  unsigned free = look(0);
  // requests: sequence n's begin at fresh[n] (of up to NEAR sequences, at begin_s[n])
  const bool near = x.N <= NEAR;
  int asked = 0;
  for (int n0 = 0; n0 < x.N; n0 += 1024) {
    const int n = n0 + tid, mine = n < x.N ? x.fresh[n] : 0;
    int total;
    const int before = scan(mine, &total);
    if (n < x.N) {
      if (near) begin_s[n] = asked + before;
      else x.fresh[n] = asked + before;
    }
    asked += total;
  }
  __syncthreads();
  auto begin = [&](int n) { return near ? begin_s[n] : x.fresh[n]; };
  // the k-th free page goes to the k-th request: to the last sequence that begins at or before k
  int given = 0;
  for (int p0 = 0; p0 < a.n_pages && given < asked; p0 += 1024 * AT_ONCE) {
    if (p0 > 0) free = look(p0);
    int total, k = scan(__builtin_popcount(free), &total);
    k += given;
    for (; free && k < asked; free &= free - 1, ++k) {
      const int p = p0 + tid * AT_ONCE + __builtin_ctz(free);
      int lo = 0, hi = x.N;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (begin(mid) <= k) lo = mid;
        else hi = mid;
      }
      const int nth = k - begin(lo);
      const int2 at = x.at[lo];
      int *entry = x.table + (size_t)lo * a.max_pages + at.x;
      if (!at.y) entry += nth;  // (its entries from there on all ask)
      else
        while (*entry != -2 - nth) ++entry;
      *entry = p;
      x.new_refs[p] = 1;
    }
    given += total;
  }
  __syncthreads();
  if (tid == 0) x.missing[0] = max(asked - given, 0);
  for (int n = tid; n < x.N; n += 1024) {
    int src = x.copies[3 * n];
    const int part = x.copies[3 * n + 2];
    const int dst = src >= 0 ? x.table[(size_t)n * a.max_pages + x.at[n].x] : -1;
    if (dst < 0) src = -1;
    x.copies[3 * n] = src;
    x.copies[3 * n + 1] = src < 0 ? -1 : dst;
    x.copies[3 * n + 2] = src < 0 ? 0 : part;
  }
  if (asked <= given) return;
  __syncthreads();
  for (size_t i = tid; i < (size_t)x.N * a.max_pages; i += 1024)
    if (x.table[i] < -1) x.table[i] = -1;
}

__global__ __launch_bounds__(kThreads) void fork_rows_kernel(Args a, Fork x)
{
  const int i0 = blockIdx.x * kThreads + threadIdx.x, lane = threadIdx.x & 63;
  for (int i = i0; i < a.n_pages; i += gridDim.x * kThreads) {
    x.new_refs[i] = x.refs[i];
    x.held[i] = 0;
  }
  const int n = __builtin_amdgcn_readfirstlane(i0 >> 6);
  if (n < x.N) fork_row(a, x, n, lane);
}
__global__ __launch_bounds__(kThreads) void fork_refs_kernel(Args a, Fork x)
{
  const int n = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * kThreads + threadIdx.x) >> 6);
  if (n < max(x.N, a.S)) fork_refs(a, x, n, threadIdx.x & 63);
}
__global__ __launch_bounds__(1024) void fork_give_kernel(Args a, Fork x) { fork_give(a, x, threadIdx.x); }
// all of it, for few sequences and pages
__global__ __launch_bounds__(1024) void fork_kernel(Args a, Fork x)
{
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  for (int i = tid; i < a.n_pages; i += 1024) {
    x.new_refs[i] = x.refs[i];
    x.held[i] = 0;
  }
  for (int n = wv; n < x.N; n += 16) fork_row(a, x, n, lane);
  __syncthreads();
  for (int n = wv; n < max(x.N, a.S); n += 16) fork_refs(a, x, n, lane);
  __threadfence();  // (the counts' atomics are done in the second-level cache: nobody reads them from the first)
  __syncthreads();
  __threadfence();
  fork_give(a, x, tid);
}

bool launch_fork(const Args &a, const Fork &x, hipStream_t st)
{
  const long most = x.N > a.S ? x.N : a.S, blocks = (most * 64 + kThreads - 1) / kThreads;
  if (!countable(blocks, kThreads)) return false;
  [&] {
    if (most <= 64 && most * a.max_pages <= 8192 && a.n_pages <= 16384) {
      BLOSSOM_LAUNCH(fork_kernel, dim3(1), dim3(1024), 0, st, a, x);
      return;
    }
    BLOSSOM_LAUNCH(fork_rows_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, st, a, x);
    BLOSSOM_LAUNCH(fork_refs_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, st, a, x);
    BLOSSOM_LAUNCH(fork_give_kernel, dim3(1), dim3(1024), 0, st, a, x);
  }();
  return true;
}

// The first `rows` positions of a page, of every key/value head, of K and of V.
__global__ __launch_bounds__(kThreads) void copy_kernel(Args a, const int *copies, int row_chunks)
{
  const int n = blockIdx.x / (2 * a.G), head = blockIdx.x - n * (2 * a.G);
  const int src = copies[3 * n], dst = copies[3 * n + 1], page = 1 << a.page_shift, rows = min(copies[3 * n + 2], page);
  if (src < 0 || src >= a.n_pages || dst < 0 || dst >= a.n_pages || src == dst) return;
  uint4 *cache = reinterpret_cast<uint4 *>(head < a.G ? a.K_cache : a.V_cache);
  const int g = head < a.G ? head : head - a.G;
  const uint4 *from = cache + ((size_t)src * a.G + g) * page * row_chunks;
  uint4 *to = cache + ((size_t)dst * a.G + g) * page * row_chunks;
  for (int i = threadIdx.x; i < rows * row_chunks; i += kThreads) to[i] = from[i];
}

bool launch_copy(const Args &a, const int *copies, int count, hipStream_t st)
{
  const long blocks = (long)count * 2 * a.G;
  if (!countable(blocks, kThreads)) return false;
  hipLaunchKernelGGL(copy_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, st, a, copies, a.d * (a.dtype == 0 ? 4 : 2) / 16);
  return true;
}

}  // namespace paged
}  // namespace blossom
