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
// reads later never lies where it wrote: keep[j] >= j > i for j > i.  No thread waits for another.  64 entries at a time, one a lane, whose
// pages are looked up together (128 trees of 33 to 64 tokens, up to 12 kept: 8.1 us, one by one 11.1, where a copy of as many rows would take
// 1; the rest is a chain of loads, length to page to row).
__global__ __launch_bounds__(kThreads) void accept_kernel(Args a, Accept x, int row_chunks)
{
  constexpr int AHEAD = 8;
  const int lane = threadIdx.x & 63;
  const int per = 2 * a.G * row_chunks, groups = (per + kThreads - 1) / kThreads;  // threads and workgroups of a sequence
  const int s = blockIdx.x / groups, at = (blockIdx.x - s * groups) * kThreads + threadIdx.x;
  const int *keep = x.keep + (size_t)s * x.width;
  const int *table = a.page_table + s * a.table_seq;
  int mine = lane < x.width ? keep[lane] : -1, last = -1;  // (requested with the lengths)
  const int first = token_at(a, s), n = max(token_at(a, s + 1) - first, 0);
  const int past = max(a.kv_len[s], 0) - n;
  const int chunk = at % row_chunks, head = min(at / row_chunks, 2 * a.G - 1);  // K's heads, then V's
  uint4 *cache = reinterpret_cast<uint4 *>(head < a.G ? a.K_cache : a.V_cache);
  const int g = head < a.G ? head : head - a.G, page = 1 << a.page_shift;
  int kept = 0;
  for (int i0 = 0; i0 < x.width; i0 += 64) {
    const int i = i0 + lane;
    if (i0 > 0) mine = i < x.width ? keep[i] : -1;
    const int up = __shfl_up(mine, 1), before = lane == 0 ? last : up;
    last = __builtin_amdgcn_readlane(mine, 63);
    const unsigned long long good = __ballot(mine > before && mine < n && mine >= 0);
    const int run = good == ~0ull ? 64 : __builtin_ctzll(~good);
    kept += run;
    // where a row of key/value head 0 lies before and after, in positions of a page times heads (below 0: it is not moved)
    auto place = [&](int pos) __attribute__((always_inline)) -> long {
      const int id = lane < run ? page_of(a, table, pos) : -1;
      return id < 0 ? -1 : ((long)id * a.G << a.page_shift) + (pos & (page - 1));
    };
    long from = mine == i ? -1 : place(past + mine);
    const long to = from < 0 ? -1 : place(past + i);
    if (to < 0) from = -1;
    unsigned long long moves = __ballot(from >= 0);
    while (moves) {
      uint4 v[AHEAD];
      uint4 *dst[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        dst[k] = nullptr;
        if (moves == 0 || at >= per) continue;
        const int l = __builtin_ctzll(moves);
        moves &= moves - 1;
        auto of = [&](long p) __attribute__((always_inline)) {
          return (long)(unsigned)__builtin_amdgcn_readlane((int)(p >> 32), l) << 32 | (unsigned)__builtin_amdgcn_readlane((int)p, l);
        };
        const long step = (long)g << a.page_shift;
        v[k] = cache[(of(from) + step) * row_chunks + chunk];
        dst[k] = cache + (of(to) + step) * row_chunks + chunk;
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (dst[k]) *dst[k] = v[k];
      if (at >= per) break;
    }
    if (run < 64) break;
  }
  if (at == 0 && x.new_len) x.new_len[s] = past + kept;
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

// Sequences take a wavefront each, which counts pages by atomics (a sum of whole numbers, in any order); fresh pages go out from one
// workgroup.  It is all chains of loads, each about a microsecond where another die wrote: 512 sequences of up to 4040 positions 18 us
// in four launches with the copies; few sequences and pages are done by one workgroup with its counts in LDS.  The eldest counts for all
// heirs (rows of 512 sequences of up to 8208 positions, pages of 8: 23.7 us, each for itself 29.6).
//
// What a new sequence takes over from q.
struct Heir {
  int len, full, part, need;  // (q < 0: nothing)
  __device__ __forceinline__ Heir(const Args &a, const Fork &x, int q)
  {
    len = q < 0 ? 0 : min(max(a.kv_len[q], 0), a.cap);
    full = len >> a.page_shift;
    part = len & ((1 << a.page_shift) - 1);
    need = q < 0 ? 0 : (int)((min((long)len + x.grow, (long)a.cap) + (1 << a.page_shift) - 1) >> a.page_shift);
  }
};
__device__ __forceinline__ int valid(const Args &a, int id) { return id >= 0 && id < a.n_pages ? id : -1; }

// New sequence n, and old sequence n, by a wavefront: its row of the new table, fresh pages as -2, -3, .. in order, how many those are, and
// which page it copies; who holds a page then, of all heirs of a parent by the eldest.  count(page, change), hold(page): of a page that a copy reads.
template <typename C, typename H>
__device__ __forceinline__ void fork_row(const Args &a, const Fork &x, int n, int lane, C &&count, H &&hold)
{
  const int mine = n < x.N ? x.parent[n] : -1, q = mine >= 0 && mine < a.S ? mine : -1;
  int heirs = 0, younger = 0;  // sequences that go on from the same parent, and that go on from old sequence n
  bool eldest = q >= 0;
  for (int i0 = 0; i0 < x.N; i0 += 64) {
    const int p = i0 + lane < x.N ? x.parent[i0 + lane] : -1;
    const unsigned long long same = __ballot(p == q && p >= 0);
    if (heirs == 0 && same) eldest = eldest && i0 + __builtin_ctzll(same) == n;
    heirs += __builtin_popcountll(same);
    younger += __builtin_popcountll(__ballot(p == n));
  }
  if (n < a.S && younger == 0) {  // dropped by all: its pages go
    const int *from = a.page_table + (size_t)n * a.max_pages;
    for (int i = lane; i < a.max_pages; i += 64) {
      const int old = valid(a, from[i]);
      if (old >= 0) count(old, -1);
    }
  }
  if (n >= x.N) return;
  const Heir h(a, x, q);
  const int *from = a.page_table + (size_t)max(q, 0) * a.max_pages;
  int *to = x.table + (size_t)n * a.max_pages;
  int fresh = 0, copy = -1, first = 0, last = -1;  // (entries that ask: how many, the first and last of them)
  const int until = eldest ? a.max_pages : h.need;
  int next = lane < until ? from[lane] : -1;
  for (int i0 = 0; i0 < a.max_pages; i0 += 64) {
    const int i = i0 + lane, old = valid(a, next);
    next = i + 64 < until ? from[i + 64] : -1;
    const bool taken = i < h.full || (i < h.need && eldest && old >= 0 && x.refs[old] == 1), asks = i < h.need && !taken;
    const unsigned long long all = __ballot(asks);
    const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(all >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)all, 0));
    if (all != 0ull) {
      if (fresh == 0) first = i0 + __builtin_ctzll(all);
      last = i0 + 63 - __builtin_clzll(all);
    }
    if (asks && i == h.full && h.part > 0) copy = old;
    if (i < a.max_pages) to[i] = taken ? old : asks ? -2 - (fresh + before) : -1;
    fresh += __builtin_popcountll(all);
    // whole pages: all heirs for the parent; of the rest the eldest lets go of what it does not take over
    const int by = i < h.full ? heirs - 1 : taken ? 0 : -1;
    if (eldest && old >= 0 && by != 0) count(old, by);
  }
  const bool apart = last - first + 1 != fresh;
  if (apart) {  // pages that are kept lie among the fresh ones: where these are
    int before = 0;
    for (int i0 = first & ~63; i0 <= last; i0 += 64) {
      const unsigned long long all = __ballot(i0 + lane <= last && to[i0 + lane] < -1);
      if (lane == 0) x.asks[(size_t)n * x.chunks + (i0 >> 6)] = make_uint4((unsigned)all, (unsigned)(all >> 32), before, 0);
      before += __builtin_popcountll(all);
    }
  }
  if (copy >= 0) hold(copy);
  const unsigned long long copies = __ballot(copy >= 0);
  copy = __builtin_amdgcn_readlane(copy, copies ? __builtin_ctzll(copies) : 0);
  if (lane == 0) {
    x.fresh[n] = fresh;
    x.len[n] = h.len;
    x.at[n] = make_int4(first, apart ? last : -1, copy, h.part);
    x.copies[3 * n] = x.copies[3 * n + 1] = -1;
    x.copies[3 * n + 2] = 0;
  }
}

// Fresh pages, by one workgroup of 1024: the k-th free page goes to the k-th request.  Pages are looked at 1024 EACH at a time, a wavefront 64 by
// 64, and listed; then every thread has a request.  (2000 free pages behind a million that are held: 200 us; 4096 pages at a time, each thread's
// own given out by itself, 512 sequences 7.6 us, so 5.8.)  An eldest's requests may lie among pages that it keeps: then fork_row leaves in x.asks
// which 64 entries at a time ask.  (Found by looking from the row's first on, 65536 pages for 64 rows took 4.8 ms, for 8 rows
// 19; so 0.08 and 0.09.)  (held_of(p): 0 if page p is free; given_out(p): it is given.)
template <int EACH, typename F, typename G>
__device__ __forceinline__ void fork_give(const Args &a, const Fork &x, int tid, F &&held_of, G &&given_out)
{
  constexpr int NEAR = 1024, WAVES = 16;
  __shared__ int sums[WAVES], begin_s[NEAR];
  __shared__ int4 at_s[NEAR];
  __shared__ unsigned short list_s[64 * EACH * WAVES];
  const int lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  // exclusive sums over the workgroup's wavefronts; *total: of all
  auto scan = [&](int upto, int *total) -> int {
    __syncthreads();
    if (lane == 63) sums[wv] = upto;
    __syncthreads();
    const int s = lane < WAVES ? sums[lane] : 0, t = wave_scan(s);
    *total = __builtin_amdgcn_readlane(t, WAVES - 1);
    return __builtin_amdgcn_readlane(t - s, wv);
  };
  // requests: sequence n's begin at fresh[n] (of up to NEAR sequences, at begin_s[n])
  const bool near = x.N <= NEAR;
  if (near && tid < x.N) at_s[tid] = x.at[tid];
  int asked = 0;
  for (int n0 = 0; n0 < x.N; n0 += 1024) {
    const int n = n0 + tid, mine = n < x.N ? x.fresh[n] : 0, upto = wave_scan(mine);
    int total;
    const int begin = asked + scan(upto, &total) + upto - mine;
    if (n < x.N) {
      if (near) begin_s[n] = begin;
      else x.fresh[n] = begin;
    }
    asked += total;
  }
  __syncthreads();
  auto begin = [&](int n) { return near ? begin_s[n] : x.fresh[n]; };
  int given = 0;
  for (int p0 = 0; p0 < a.n_pages && given < asked; p0 += 64 * EACH * WAVES) {
    unsigned long long free[EACH];
    int mine = 0, total, held[EACH];
    const int first = p0 + 64 * EACH * wv + lane;
    if (first - lane < a.n_pages) {
#pragma unroll
      for (int k = 0; k < EACH; ++k) held[k] = held_of(min(first + 64 * k, a.n_pages - 1));
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      free[k] = first - lane < a.n_pages ? __ballot(first + 64 * k < a.n_pages && held[k] == 0) : 0ull;
      mine += __builtin_popcountll(free[k]);
    }
    int at = scan(mine, &total);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      if (free[k] >> lane & 1ull)
        list_s[at + __builtin_amdgcn_mbcnt_hi((unsigned)(free[k] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)free[k], 0))] = (unsigned short)(64 * (EACH * wv + k) + lane);
      at += __builtin_popcountll(free[k]);
    }
    __syncthreads();
    for (int r = tid; r < min(total, asked - given); r += 1024) {
      const int p = p0 + list_s[r], k = given + r;
      int lo = 0, hi = x.N;  // the last sequence whose requests begin at or before k
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (begin(mid) <= k) lo = mid;
        else hi = mid;
      }
      const int nth = k - begin(lo);
      const int4 at = near ? at_s[lo] : x.at[lo];
      int i = at.x;
      int *row = x.table + (size_t)lo * a.max_pages;
      if (at.y < 0) i += nth;
      else {  // the last 64 entries before which no more than nth ask, and of those that ask here the one
        int c = at.x >> 6, end = (at.y >> 6) + 1;
        const uint4 *asks = x.asks + (size_t)lo * x.chunks;
        while (end - c > 1) {
          const int mid = (c + end) >> 1;
          if ((int)asks[mid].z <= nth) c = mid;
          else end = mid;
        }
        const uint4 here = asks[c];
        unsigned long long all = (unsigned long long)here.y << 32 | here.x;
        for (int left = nth - (int)here.z; left > 0; --left) all &= all - 1;
        i = 64 * c + __builtin_ctzll(all);
      }
      row[i] = p;
      given_out(p);
      if (i == at.x && at.z >= 0) {
        x.copies[3 * lo] = at.z;
        x.copies[3 * lo + 1] = p;
        x.copies[3 * lo + 2] = at.w;
      }
    }
    given += total;
  }
  if (tid == 0) x.missing[0] = max(asked - given, 0);
  if (asked <= given) return;
  __syncthreads();
  for (size_t i = tid; i < (size_t)x.N * a.max_pages; i += 1024)
    if (x.table[i] < -1) x.table[i] = -1;
}

__global__ __launch_bounds__(kThreads) void fork_begin_kernel(Args a, Fork x)
{
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.n_pages) return;
  x.new_refs[i] = x.refs[i];
  x.held[i] = 0;
}
__global__ __launch_bounds__(kThreads) void fork_rows_kernel(Args a, Fork x)
{
  const int n = __builtin_amdgcn_readfirstlane((int)((blockIdx.x * kThreads + threadIdx.x) >> 6));
  if (n < max(x.N, a.S))
    fork_row(a, x, n, threadIdx.x & 63, [&](int p, int by) { atomicAdd(x.new_refs + p, by); }, [&](int p) { x.held[p] = 1; });
}
__global__ __launch_bounds__(1024) void fork_give_kernel(Args a, Fork x)
{
  fork_give<16>(
      a, x, threadIdx.x,
      [&](int p) { return x.new_refs[p] | x.held[p]; },
      [&](int p) { x.new_refs[p] = 1; });
}
// all of it, for few sequences and pages
constexpr int kFewPages = 8192, kFewForks = 64;
constexpr int kMostForks = 1 << 20;  // sequences: each looks through the parents of all
__global__ __launch_bounds__(1024) void fork_kernel(Args a, Fork x)
{
  __shared__ int refs_s[kFewPages];
  __shared__ unsigned held_s[kFewPages / 32];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  for (int i = tid; i < a.n_pages; i += 1024) refs_s[i] = x.refs[i];
  if (tid < kFewPages / 32) held_s[tid] = 0;
  __syncthreads();
  for (int n = wv; n < max(x.N, a.S); n += 16)
    fork_row(a, x, n, lane, [&](int p, int by) { atomicAdd(refs_s + p, by); }, [&](int p) { atomicOr(held_s + (p >> 5), 1u << (p & 31)); });
  __syncthreads();
  fork_give<4>(
      a, x, tid,
      [&](int p) { return refs_s[p] | (int)(held_s[p >> 5] >> (p & 31) & 1u); },
      [&](int p) { refs_s[p] = 1; });
  __syncthreads();
  for (int i = tid; i < a.n_pages; i += 1024) x.new_refs[i] = refs_s[i];
}

bool launch_fork(const Args &a, const Fork &x, hipStream_t st)
{
  const long most = x.N > a.S ? x.N : a.S, rows = (most * 64 + kThreads - 1) / kThreads, pages = ((long)a.n_pages + kThreads - 1) / kThreads;
  if (most > kMostForks || a.n_pages > 1 << 30) return false;  // (pages are counted past the last)
  [&] {
    if (most <= kFewForks && most * a.max_pages <= 8192 && a.n_pages <= kFewPages) {
      BLOSSOM_LAUNCH(fork_kernel, dim3(1), dim3(1024), 0, st, a, x);
      return;
    }
    BLOSSOM_LAUNCH(fork_begin_kernel, dim3((unsigned)pages), dim3(kThreads), 0, st, a, x);
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
