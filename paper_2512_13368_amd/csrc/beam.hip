// Beam search's selection: of every history's W beams and V items the K best continuations, by the beam's score and the item's
// log-probability,  score + logit - log sum exp(logits of the row).
//
// Scores of two beams may lie as near to each other as rounding lets them, and which of them is chosen is a whole number: sums of
// exponentials and scores are held in 64 bits.  Candidates are ordered by score, then beam, then logit, then item (the lower one first),
// which is one order whatever the workgroups do.
//   rows_kernel   a workgroup takes a run of a row: its sum, and its K best logits
//   merge_kernel  a workgroup a history: sums joined, then the K best of the runs' lists
#include "beam.h"

#include "common.h"
#include "launch.h"

namespace blossom {
namespace beam {

namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 64;   // groups of 4 lanes, whose largest logits give a bound that K logits reach
constexpr int kList = 1024;   // logits beyond the bound that are kept at a time
typedef unsigned long long u64;

// logits and items as one number: the larger logit first, then the lower item.  0: none.
__device__ __forceinline__ unsigned ordered(float x)
{
  const unsigned b = __float_as_uint(x + 0.0f);  // (-0 is 0)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(unsigned o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ u64 key_of(float x, int item) { return (u64)ordered(x) << 32 | (unsigned)~item; }
__device__ __forceinline__ int item_of(u64 key) { return (int)~(unsigned)key; }
__device__ __forceinline__ u64 ordered(double x)
{
  const u64 b = (u64)__double_as_longlong(x + 0.0);
  return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double score_of(u64 o) { return __longlong_as_double((long long)(o >> 63 ? o ^ 1ull << 63 : ~o)); }

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(bf16_t x) { return __uint_as_float((unsigned)x.bits << 16); }

// is (p, w, k) before (q, v, l): score, beam, logit and item?
__device__ __forceinline__ bool before(u64 p, int w, u64 k, u64 q, int v, u64 l) { return p != q ? p > q : w != v ? w < v : k > l; }

}  // namespace

// Block `lists` of a row: a run of `subs` pieces of kThreads * LD * 16 bytes.
template <typename T, int LD>
__global__ __launch_bounds__(kThreads) void rows_kernel(Args a, int subs)
{
  constexpr int VEC = 16 / (int)sizeof(T), EL = LD * VEC, SUB = kThreads * EL;
  struct __attribute__((packed, aligned(sizeof(T)))) Piece { T x[VEC]; };  // (rows begin at any element)
  __shared__ u64 list[kList + kMost], best[kMost];
  __shared__ float group_s[kGroups], wave_s[4];
  __shared__ double sum_s[4];
  __shared__ u64 top_s[4];
  __shared__ int count_s;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x / a.lists, run = blockIdx.x - row * a.lists;
  const float score = a.score[row];
  const bool off = (a.ended && a.ended[row]) || !(score > -INFINITY);  // goes on in one way, or not at all
  const T *x0 = static_cast<const T *>(a.logits) + row * a.stride;
  const long lo = (long)run * subs * SUB, hi = off ? lo : lo + (long)subs * SUB < a.V ? lo + (long)subs * SUB : a.V;
  float m = -INFINITY;
  double s = 0.0;
  int have = 0;
  for (long at = lo; at < hi; at += SUB) {
    float x[EL];
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < LD; ++j) {
      const long i = at + (long)(j * kThreads + tid) * VEC;
      if (i + VEC <= a.V) {
        const Piece p = *reinterpret_cast<const Piece *>(x0 + i);
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[j * VEC + e] = as_float(p.x[e]);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[j * VEC + e] = i + e < a.V ? as_float(x0[i + e]) : -INFINITY;
      }
    }
#pragma unroll
    for (int e = 0; e < EL; ++e) {
      x[e] = x[e] == x[e] ? x[e] : -INFINITY;  // (a NaN counts as an item that is ruled out)
      top = fmaxf(top, x[e]);
    }
    // ---- a bound that K logits reach: the K-th largest of the groups' largest, or the K-th best so far ----
    float group = fmaxf(top, __shfl_xor(top, 1));
    group = fmaxf(group, __shfl_xor(group, 2));
    if ((lane & 3) == 0) group_s[16 * wv + (lane >> 2)] = group;
    if (tid == 0) count_s = 0;
    __syncthreads();
    const float mine = group_s[lane];
    int rank = 0;
    for (int i = 0; i < kGroups; ++i) {
      const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), i));
      rank += o > mine || (o == mine && i < lane);
    }
    const float m_new = fmaxf(m, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), __builtin_ctzll(__ballot(rank == 0)))));
    const float bound = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), __builtin_ctzll(__ballot(rank == min(a.K, kGroups) - 1))));
    u64 least = max((u64)ordered(bound), (u64)ordered(-INFINITY) + 1) << 32;  // (-inf is no candidate)
    if (have == a.K) least = max(least, best[a.K - 1] + 1);
#pragma unroll
    for (int j = 0; j < LD; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const u64 key = key_of(x[j * VEC + e], (int)(at + (long)(j * kThreads + tid) * VEC + e));
        if (key >= least) {
          const int to = atomicAdd(&count_s, 1);
          if (to < kList) list[to] = key;
        }
      }
    __syncthreads();
    int n = count_s;
    if (n > kList) {  // (as many as that where logits are equal, or lie in the same lanes' places): one after another
      u64 last = ~0ull;
      for (n = 0; n < a.K; ++n) {
        u64 k = 0;
#pragma unroll
        for (int j = 0; j < LD; ++j)
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const u64 key = key_of(x[j * VEC + e], (int)(at + (long)(j * kThreads + tid) * VEC + e));
            if (key >= least && key < last && key > k) k = key;
          }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) k = max(k, (u64)__shfl_xor((long long)k, o));
        __syncthreads();
        if (lane == 0) top_s[wv] = k;
        __syncthreads();
        last = max(max(top_s[0], top_s[1]), max(top_s[2], top_s[3]));
        if (last == 0) break;
        if (tid == 0) list[n] = last;
      }
    }
    if (tid < have) list[n + tid] = best[tid];
    __syncthreads();
    n += have;
    for (int i = tid; i < n; i += kThreads) {
      const u64 k = list[i];
      int r = 0;
      for (int j = 0; j < n; ++j) r += list[j] > k;
      if (r < a.K) best[r] = k;
    }
    have = min(n, a.K);
    // ---- the sum ----
    if (m_new > -INFINITY && m_new < INFINITY) {
      if (m_new > m) s *= exp((double)m - (double)m_new);
#pragma unroll
      for (int e = 0; e < EL; ++e) s += exp((double)x[e] - (double)m_new);
    }
    m = m_new;
    __syncthreads();
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
  if (lane == 0) sum_s[wv] = s;
  __syncthreads();
  if (tid == 0) a.stats[blockIdx.x] = make_double2((double)m, (sum_s[0] + sum_s[1]) + (sum_s[2] + sum_s[3]));
  if (tid < a.K) a.lists_of[(size_t)blockIdx.x * a.K + tid] = tid < have ? best[tid] : 0;
}

__global__ __launch_bounds__(kThreads) void merge_kernel(Args a)
{
  constexpr int PAIRS = kMost * (kMost + 1) / 2;
  __shared__ double lse_s[kMost];
  __shared__ u64 head_s[kLists], logit_s[kLists], group_s[kGroups];
  __shared__ int near_s[kLists], chosen_s[kMost], count_s[2];
  __shared__ u64 p_s[PAIRS], k_s[PAIRS];
  __shared__ unsigned char w_s[PAIRS];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
  const int L = a.W * a.lists;
  const size_t row0 = (size_t)b * a.W;
  if (tid < 2) count_s[tid] = 0;
  // ---- log sum exp of each beam's row ----
  for (int w = wv; w < a.W; w += 4) {
    const double2 *st = a.stats + (row0 + w) * a.lists;
    double m = -INFINITY;
    for (int i = lane; i < a.lists; i += 64) m = fmax(m, st[i].x);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = fmax(m, __shfl_xor(m, o));
    double s = 0.0;
    for (int i = lane; i < a.lists; i += 64) s += st[i].x > -INFINITY ? st[i].y * exp(st[i].x - m) : 0.0;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) lse_s[w] = m == INFINITY ? INFINITY : m + log(s);
  }
  __syncthreads();
  // place of element j of list l in the order: its score, and its logit and item; none: 0
  auto look = [&](int l, int j, u64 *k) -> u64 {
    const int w = l / a.lists;
    const double score = (double)a.score[row0 + w];
    double to;
    if (a.ended && a.ended[row0 + w]) {
      *k = key_of(0.0f, a.eos);
      to = l == w * a.lists && j == 0 ? score : -INFINITY;
    } else {
      *k = a.lists_of[(row0 * a.lists + l) * a.K + j];
      to = *k == 0 ? -INFINITY : score + ((double)logit_of((unsigned)(*k >> 32)) - lse_s[w]);
    }
    return to > -INFINITY ? ordered(to) : 0;  // (a NaN neither)
  };
  // ---- lists whose first element may be among the K best: the K best first elements ----
  u64 top = 0;
  for (int l = tid; l < L; l += kThreads) {
    u64 k;
    const u64 p = look(l, 0, &k);
    head_s[l] = p;
    logit_s[l] = k;
    top = max(top, p);
  }
  top = max(top, (u64)__shfl_xor((long long)top, 1));
  top = max(top, (u64)__shfl_xor((long long)top, 2));
  if ((lane & 3) == 0) group_s[16 * wv + (lane >> 2)] = top;
  __syncthreads();
  u64 bound;
  {
    const u64 mine = group_s[lane];
    int rank = 0;
    for (int i = 0; i < kGroups; ++i) rank += group_s[i] > mine || (group_s[i] == mine && i < lane);
    const int at = __builtin_ctzll(__ballot(rank == min(a.K, kGroups) - 1));
    bound = max(group_s[at], 1ull);
  }
  for (int l = tid; l < L; l += kThreads)
    if (head_s[l] >= bound) near_s[atomicAdd(&count_s[0], 1)] = l;
  __syncthreads();
  const int n_near = count_s[0], n_lists = min(n_near, a.K);
  for (int i = tid; i < n_near; i += kThreads) {
    const int l = near_s[i], w = l / a.lists;
    int r = 0;
    for (int j = 0; j < n_near; ++j) {
      const int o = near_s[j];
      r += before(head_s[o], o / a.lists, logit_s[o], head_s[l], w, logit_s[l]);
    }
    if (r < a.K) chosen_s[r] = l;
  }
  __syncthreads();
  // ---- element j of the r-th of them has r + j before it ----
  const int last = n_lists == a.K ? chosen_s[a.K - 1] : -1;
  for (int i = tid; i < n_lists * a.K; i += kThreads) {
    const int r = i / a.K, j = i - r * a.K;
    if (r + j >= a.K) continue;
    const int l = chosen_s[r], w = l / a.lists;
    u64 k;
    const u64 p = look(l, j, &k);
    if (p == 0 || (last >= 0 && l != last && !before(p, w, k, head_s[last], last / a.lists, logit_s[last]))) continue;
    const int to = atomicAdd(&count_s[1], 1);
    p_s[to] = p; k_s[to] = k; w_s[to] = (unsigned char)w;
  }
  __syncthreads();
  const int n = count_s[1];
  const size_t out = (size_t)b * a.K;
  for (int i = tid; i < n; i += kThreads) {
    const u64 p = p_s[i], k = k_s[i];
    const int w = w_s[i];
    int r = 0;
    for (int j = 0; j < n; ++j) r += before(p_s[j], w_s[j], k_s[j], p, w, k);
    if (r >= a.K) continue;
    const int item = item_of(k);
    a.parent[out + r] = (int)(row0 + w);
    a.token[out + r] = item;
    a.out_score[out + r] = (float)score_of(p);
    if (a.out_ended) a.out_ended[out + r] = item == a.eos || (a.ended && a.ended[row0 + w]);
  }
  for (int r = n + tid; r < a.K; r += kThreads) {
    a.parent[out + r] = a.token[out + r] = -1;
    a.out_score[out + r] = -INFINITY;
    if (a.out_ended) a.out_ended[out + r] = 0;
  }
}

namespace {

int piece(int dtype, int loads) { return kThreads * loads * (dtype == 0 ? 4 : 8); }

}  // namespace

void plan(Args &a)
{
  const long rows = (long)a.B * a.W;
  a.loads = 8;
  if (rows * (((long)a.V + piece(a.dtype, 8) - 1) / piece(a.dtype, 8)) < 1024) a.loads = 2;
  const long pieces = ((long)a.V + piece(a.dtype, a.loads) - 1) / piece(a.dtype, a.loads);
  const long want = (2048 + rows - 1) / rows, most = kLists / a.W;
  long lists = pieces < want ? pieces : want;
  if (lists > most) lists = most;
  a.subs = (int)((pieces + lists - 1) / lists);
  a.lists = (int)((pieces + a.subs - 1) / a.subs);
}

bool launch(const Args &a, hipStream_t st)
{
  const long blocks = (long)a.B * a.W * a.lists;
  if (blocks * kThreads >= 1l << 32) return false;
  const dim3 grid((unsigned)blocks), block(kThreads);
  [&] {
    if (a.dtype == 0 && a.loads == 8) BLOSSOM_LAUNCH((rows_kernel<float, 8>), grid, block, 0, st, a, a.subs);
    else if (a.dtype == 0) BLOSSOM_LAUNCH((rows_kernel<float, 2>), grid, block, 0, st, a, a.subs);
    else if (a.loads == 8) BLOSSOM_LAUNCH((rows_kernel<bf16_t, 8>), grid, block, 0, st, a, a.subs);
    else BLOSSOM_LAUNCH((rows_kernel<bf16_t, 2>), grid, block, 0, st, a, a.subs);
    BLOSSOM_LAUNCH(merge_kernel, dim3((unsigned)a.B), block, 0, st, a);
  }();
  return true;
}

}  // namespace beam
}  // namespace blossom
