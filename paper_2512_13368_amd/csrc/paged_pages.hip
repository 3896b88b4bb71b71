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

// refs go over, and who is the eldest
__global__ __launch_bounds__(kThreads) void fork_begin_kernel(Args a, Fork x)
{
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i < a.n_pages) {
    x.new_refs[i] = x.refs[i];
    x.held[i] = 0;
  }
  if (i < a.S) {
    int e = x.N;
    for (int n = 0; n < x.N; ++n)
      if (x.parent[n] == i) {
        e = n;
        break;
      }
    x.eldest[i] = e;
  }
}

// rows of the new table, and what changes hands
__global__ __launch_bounds__(kThreads) void fork_rows_kernel(Args a, Fork x)
{
  __shared__ int fresh_s;
  const int b = blockIdx.x, tid = threadIdx.x;
  if (b < x.N) {
    const Heir h(a, x, b);
    const bool eldest = h.q >= 0 && x.eldest[h.q] == b;
    const int *from = a.page_table + (size_t)max(h.q, 0) * a.max_pages;
    int *to = x.table + (size_t)b * a.max_pages;
    if (tid == 0) fresh_s = 0;
    __syncthreads();
    int copy = -1;
    for (int i = tid; i < a.max_pages; i += kThreads) {
      int id = -1;
      if (i < h.need) {
        const int old = valid(a, from[i]);
        if (i < h.full) {
          id = old;
        } else if (eldest && old >= 0 && x.refs[old] == 1) {
          id = old;
        } else {
          atomicAdd(&fresh_s, 1);
          if (i == h.full && h.part > 0) copy = old;
        }
        if (id >= 0 && !eldest) atomicAdd(x.new_refs + id, 1);
        if (i == h.full && h.part > 0) {
          if (copy >= 0) atomicAdd(x.held + copy, 1);
          x.copies[3 * b] = copy;
        }
      }
      to[i] = id;
    }
    if (tid == 0 && !(h.part > 0 && h.full < h.need)) x.copies[3 * b] = -1;
    __syncthreads();
    if (tid == 0) {
      x.fresh[b] = fresh_s;
      x.len[b] = h.len;
    }
  }
  if (b < a.S) {  // what nobody, or the eldest, does not take over
    const int e = x.eldest[b];
    const int *from = a.page_table + (size_t)b * a.max_pages;
    Heir h(a, x, min(e, x.N - 1));
    if (e >= x.N) h.full = h.need = 0;
    for (int i = tid; i < a.max_pages; i += kThreads) {
      const int old = valid(a, from[i]);
      if (old < 0 || i < h.full || (i < h.need && x.refs[old] == 1)) continue;
      atomicSub(x.new_refs + old, 1);
    }
  }
}

// fresh pages, by one workgroup
__global__ __launch_bounds__(1024) void fork_give_kernel(Args a, Fork x)
{
  __shared__ int sums[16], total_s;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  // exclusive sums over the workgroup; *total: of all
  auto scan = [&](int v, int *total) -> int {
    const int upto = wave_scan(v);
    __syncthreads();
    if (lane == 63) sums[wv] = upto;
    __syncthreads();
    if (wv == 0) {
      const int s = lane < 16 ? sums[lane] : 0, t = wave_scan(s);
      if (lane < 16) sums[lane] = t - s;
      if (lane == 15) total_s = t;
    }
    __syncthreads();
    *total = total_s;
    return sums[wv] + upto - v;
  };
  // requests: sequence n's begin at fresh[n]
  int asked = 0;
  for (int n0 = 0; n0 < x.N; n0 += 1024) {
    const int n = n0 + tid, mine = n < x.N ? x.fresh[n] : 0;
    int total;
    const int before = scan(mine, &total);
    if (n < x.N) x.fresh[n] = asked + before;
    asked += total;
  }
  __syncthreads();
  // the k-th free page goes to the k-th request: to the last sequence that begins at or before k
  int given = 0;
  for (int p0 = 0; p0 < a.n_pages && given < asked; p0 += 1024) {
    const int p = p0 + tid;
    const bool free = p < a.n_pages && x.new_refs[p] == 0 && x.held[p] == 0;
    int total;
    const int k = given + scan(free, &total);
    if (free && k < asked) {
      int lo = 0, hi = x.N;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (x.fresh[mid] <= k) lo = mid;
        else hi = mid;
      }
      // its (k - fresh[lo])-th entry without a page
      const Heir h(a, x, lo);
      int *row = x.table + (size_t)lo * a.max_pages;
      const int *from = a.page_table + (size_t)h.q * a.max_pages;
      const bool eldest = x.eldest[h.q] == lo;
      int at = k - x.fresh[lo], i = h.full;
      for (; i < h.need; ++i) {
        const int old = valid(a, from[i]);
        if (!(eldest && old >= 0 && x.refs[old] == 1) && at-- == 0) break;
      }
      row[i] = p;
      x.new_refs[p] = 1;
    }
    given += total;
  }
  __syncthreads();
  if (tid == 0) x.missing[0] = max(asked - given, 0);
  for (int n = tid; n < x.N; n += 1024) {
    const Heir h(a, x, n);
    const int src = x.copies[3 * n], dst = src >= 0 ? x.table[(size_t)n * a.max_pages + h.full] : -1;
    const bool on = src >= 0 && dst >= 0;
    x.copies[3 * n] = on ? src : -1;
    x.copies[3 * n + 1] = on ? dst : -1;
    x.copies[3 * n + 2] = on ? h.part : 0;
  }
}

bool launch_fork(const Args &a, const Fork &x, hipStream_t st)
{
  const long begin = ((long)(a.n_pages > a.S ? a.n_pages : a.S) + kThreads - 1) / kThreads, rows = x.N > a.S ? x.N : a.S;
  if (!countable(begin, kThreads) || !countable(rows, kThreads)) return false;
  [&] {
    BLOSSOM_LAUNCH(fork_begin_kernel, dim3((unsigned)begin), dim3(kThreads), 0, st, a, x);
    BLOSSOM_LAUNCH(fork_rows_kernel, dim3((unsigned)rows), dim3(kThreads), 0, st, a, x);
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
