// Beam search's selection: of every history's W beams and V items the K best continuations, by the beam's score and the item's
// log-probability,  score + logit - log sum exp(logits of the row).
//
// Scores of two beams may lie as near to each other as rounding lets them, and which of them is chosen is a whole number: sums of
// exponentials and scores are held in 64 bits.  Candidates are ordered by score, then beam, then logit, then item (the lower one first),
// which is one order whatever the workgroups do.
//   rows_kernel   a workgroup takes a run of a row: its sum, and its K best logits
//   merge_kernel  a workgroup a history: sums joined, then the K best of the runs' lists
//   few_kernel    both, for histories of few logits
#include "beam.h"

#include <type_traits>

#include "common.h"
#include "launch.h"

namespace blossom {
namespace beam {

namespace {

constexpr int kWaves = 8;     // of a run
constexpr int kFewLogits = 8192;  // of a history that one workgroup may take by itself (see plan)
constexpr int kFewCandidates = 1024;  // in the lists of a history: four a thread of the merge's small workgroup
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

// is (p, w, k) before (q, v, l): score, beam, logit and item?
__device__ __forceinline__ bool before(u64 p, int w, u64 k, u64 q, int v, u64 l) 
{
  return (p > q) | ((p == q) & ((w < v) | ((w == v) & (k > l))));  // (without branches)
}

}  // namespace

// The sum of 2^t[i] in 64 bits for |t| <= 1000: the whole part goes to the exponent, the rest f in [-1/2, 1/2] through the polynomial of
// degree 8 that meets 2^f at Chebyshev's nine points (relative error 1.1e-12 at most; half a unit of an fp32 score is 6e-8 of it).  N at
// a time, for one alone is a chain of 14 instructions that wait for each other.
template <int N>
__device__ __forceinline__ double exp2_sum(const double (&t)[N])
{
  typedef unsigned pair __attribute__((ext_vector_type(2)));
  constexpr double kShift = 6755399441055744.0;  // 1.5 * 2^52: a sum with it has the whole part in its low bits
  constexpr double c[9] = {1.0, 0.69314718054593349, 0.24022650695812989, 0.055504109412059341, 0.0096181291594026191, 0.0013333450567999659,
                           0.00015403455852411408, 1.5310079402479794e-05, 1.3255224887698904e-06};
  double at[N], f[N], p[N];
#pragma unroll
  for (int i = 0; i < N; ++i) at[i] = t[i] + kShift;
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = at[i] - kShift;
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = t[i] - f[i];
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = fma(c[8], f[i], c[7]);
#pragma unroll
  for (int k = 6; k >= 0; --k) {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = fma(p[i], f[i], c[k]);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    pair w = __builtin_bit_cast(pair, p[i]);
    w.y += __builtin_bit_cast(pair, at[i]).x << 20;
    p[i] = __builtin_bit_cast(double, w);
  }
#pragma unroll
  for (int k = N / 2; k >= 1; k /= 2)
#pragma unroll
    for (int i = 0; i < k; ++i) p[i] += p[i + k];
  return p[0];
}

constexpr double kLog2e = 1.4426950408889634;
constexpr double kLeastExp = -690.0;  // e^-690 of a sum that is 1 or more: nothing
// (x - m) log2 e for x <= m, m finite, from e^-690 on (x that is -inf or NaN: that).  The difference is taken in 64 bits, where it is exact or far
// below -690.
__device__ __forceinline__ double log2_from(double x, double m) { return fmax(x - m, kLeastExp) * kLog2e; }
__device__ __forceinline__ double exp_from(double x, double m)
{
  const double t[1] = {log2_from(x, m)};
  return exp2_sum(t);
}
// The same as one product and sum, for many logits by one m near 0 (up to kNear: m log2 e is off by 2^-41, and a 32-bit m - 690 by 2^-12).
// (Farther, m log2 e would be off by as much as differences are, and m - 690 be m.)
constexpr float kNear = 4096.0f;
struct FromNear {
  float least;
  double ref;
  __device__ __forceinline__ explicit FromNear(float m) : least(m + (float)kLeastExp), ref(-(double)m * kLog2e) {}
  __device__ __forceinline__ double log2(float x) const { return fma((double)(x > least ? x : least), kLog2e, ref); }
};

__device__ __forceinline__ float element(const float *p) { return *p; }
__device__ __forceinline__ float element(const bf16_t *p) { return __uint_as_float((unsigned)p->bits << 16); }

// 16 bytes of a row, as its elements
template <typename T>
struct Piece;
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float get(const uint4 &v, int e) { return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w); }
};
template <>
struct Piece<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float get(const uint4 &v, int e)
  {
    const unsigned w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
    return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
  }
};

// e^x of bf16 logits from a table in LDS: all 2560 with 2^-14 <= |x| < 64 of either sign, at 1 + (code - that of 2^-14); at 0 what is nearer
// to 0 (1, to which x + x^2/2 is added: e^x to 2^-42/6), at the end what is larger (nothing: the sum of a piece whose largest logit
// lies between -20 and 64 does not miss e^-64; other pieces go by the polynomial).  Of two logits in a register the places take eight instructions, where the
// polynomial takes 36: 512 rows of 152063 logits 82 us by the polynomial, 36 so (other things changed with it); a quarter of them by the
// polynomial, which leaves LDS less to do, 42.  Rows that lie elsewhere are slower by that: with 40 or 100 taken from every logit, or 70 added,
// the selection from 512 rows takes 70 to 73 us where it takes 45.
constexpr int kLeast = (127 - 14) << 7;
struct Table {
  static constexpr int kEnd = ((127 + 6) << 7) - kLeast + 1;  // the place of what is larger
  static constexpr int kSign = 4096, kSize = kSign + kEnd + 1;  // places of the negative ones begin at kSign
  static_assert(kEnd < kSign && kSign * sizeof(double) == 1 << 15, "");
  static __device__ __forceinline__ void fill(double *to, int tid, int threads)
  {
    for (int i = tid; i < 2 * (kEnd + 1); i += threads) {
      const bool minus = i > kEnd;
      const int at = minus ? i - (kEnd + 1) : i;
      const float x = __uint_as_float((unsigned)(at - 1 + kLeast) << 16 | (minus ? 0x80000000u : 0u));
      const double t[1] = {(double)(at == 0 || at >= kEnd ? 0.0f : x) * kLog2e};
      to[minus ? kSign + at : at] = at >= kEnd ? 0.0 : exp2_sum(t);
    }
  }
  // the sum over 16 bytes of logits
  static __device__ __forceinline__ double sum(const double *table, const uint4 &v)
  {
    typedef unsigned short two __attribute__((ext_vector_type(2)));
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
    const two below = {kLeast - 1, kLeast - 1}, end = {kEnd, kEnd}, three = {3, 3};
    const char *bytes = reinterpret_cast<const char *>(table);
    two least = end;
    double e[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const two at = __builtin_elementwise_min(__builtin_elementwise_sub_sat(__builtin_bit_cast(two, w[i] & 0x7FFF7FFFu), below), end);
      least = __builtin_elementwise_min(least, at);
      const unsigned place = __builtin_bit_cast(unsigned, at << three) | (w[i] & 0x80008000u);  // in bytes: a logit's sign is that of kSign
      e[2 * i] = *reinterpret_cast<const double *>(bytes + (place & 0xFFFFu));
      e[2 * i + 1] = *reinterpret_cast<const double *>(bytes + (place >> 16));
    }
#pragma unroll
    for (int k = 4; k >= 1; k /= 2)
#pragma unroll
      for (int i = 0; i < k; ++i) e[i] += e[i + k];
    if (__any(least.x == 0 || least.y == 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = Piece<bf16_t>::get(v, i);
        const double y = fabsf(x) < 0x1p-14f ? (double)x : 0.0;
        e[0] = fma(y, fma(y, 0.5, 1.0), e[0]);
      }
    }
    return e[0];
  }
};

// A wavefront's best logits are held as keys in LDS, in no order until they are more than fit: then, and after every piece, the K best
// are kept.
constexpr int kHold = 2 * kMost;

// Leaves the K best of n keys, in order, and returns how many there are.  (One wavefront's LDS: no other touches it.)
__device__ __forceinline__ int keep_best(u64 *keys, int n, int K, int lane)
{
  u64 mine[kHold / 64];
  int rank[kHold / 64];
  auto some = [&](auto rounds) __attribute__((always_inline)) {
    constexpr int R = decltype(rounds)::value;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mine[r] = 64 * r + lane < n ? keys[64 * r + lane] : 0;
      rank[r] = 0;
    }
    for (int j = 0; j < n; ++j) {
      const u64 o = keys[j];
#pragma unroll
      for (int r = 0; r < R; ++r) rank[r] += o > mine[r];
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (64 * r + lane < n && rank[r] < K) keys[rank[r]] = mine[r];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  if (n <= 64) some(std::integral_constant<int, 1>{});
  else some(std::integral_constant<int, kHold / 64>{});
  return min(n, K);
}

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

// Workgroup (row, run) takes `subs` pieces of the row, its wavefronts one after another: of 64 * LD * 16 bytes each, the next on its way
// while one is worked on.  A lane keeps the sum and the largest of its logits.  When the run is done, the K-th largest of 64 groups' largest
// bounds what may be among the K best: the few lanes that reach it have their loads looked at again.
template <typename T, int LD, bool TABLE>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(4))) void rows_kernel(Args a)
{
  typedef Piece<T> P;
  constexpr int VEC = P::N, SUB = 64 * LD * VEC, THREADS = 64 * kWaves, FOUND = kWaves * kHold;
  static_assert(!TABLE || sizeof(T) == 2, "");
  struct __attribute__((packed, aligned(sizeof(T)))) Any { uint4 v; };  // (rows begin at any element)
  __shared__ u64 held[kWaves][kHold];
  __shared__ double table[TABLE ? Table::kSize : 1];
  __shared__ double sum_s[kWaves];
  __shared__ float top_s[kWaves], group_s[kWaves][64];
  __shared__ int count_s[2], have_s[kWaves];
  __shared__ unsigned bound_s;
  __shared__ unsigned short lane_s[THREADS];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x / a.lists, run = blockIdx.x - row * a.lists;
  const float score = a.score[row];
  const bool off = (a.ended && a.ended[row]) || !(score > -INFINITY);  // goes on in one way, or not at all
  const T *x0 = static_cast<const T *>(a.logits) + row * a.stride;
  const long begin = (long)run * a.subs * SUB, end = off ? begin : begin + (long)a.subs * SUB < a.V ? begin + (long)a.subs * SUB : a.V;
  auto get = [&](long i) __attribute__((always_inline)) -> uint4 {
    if (i + VEC <= a.V) return reinterpret_cast<const Any *>(x0 + i)->v;
    // the row's end: what is not there is ruled out
    constexpr int BITS = 8 * sizeof(T);
    constexpr u64 kNone = sizeof(T) == 4 ? 0xFF800000FF800000ull : 0xFF80FF80FF80FF80ull;
    u64 w[2] = {kNone, kNone};
#pragma unroll 1
    for (int e = 0; i + e < a.V; ++e) {
      const u64 b = (u64)(__float_as_uint(element(x0 + i + e)) >> (32 - BITS));
      const int to = BITS * e & 63;
      const u64 clear = ~(((1ull << BITS) - 1ull) << to);
      if (BITS * e < 64) w[0] = (w[0] & clear) | b << to;
      else w[1] = (w[1] & clear) | b << to;
    }
    return make_uint4((unsigned)w[0], (unsigned)(w[0] >> 32), (unsigned)w[1], (unsigned)(w[1] >> 32));
  };
  uint4 next[LD];
  auto load = [&](long at) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < LD; ++j) next[j] = get(at + (j * 64 + lane) * VEC);
  };
  float m = -INFINITY, lane_top = -INFINITY;
  double s = 0.0, plain = 0.0;  // sums by reference m, and by none: of what the table gives
  long at = begin + wv * SUB;
  if (at < end) load(at);
  if (tid < 2) count_s[tid] = 0;
  if constexpr (TABLE) {
    if (!off) Table::fill(table, tid, THREADS);
    __syncthreads();
  }
  for (; at < end; at += kWaves * SUB) {
    uint4 v[LD];
#pragma unroll
    for (int j = 0; j < LD; ++j) v[j] = next[j];
    if (at + kWaves * SUB < end) load(at + kWaves * SUB);
    // (a NaN counts as an item that is ruled out: fmaxf takes the other)
    float top = -INFINITY;
    bool exact = true;
    if constexpr (sizeof(T) == 2) {  // of bf16 the largest as 16-bit whole numbers, two at once, where that is one above 0 and no NaN
      typedef short two __attribute__((ext_vector_type(2)));
      two most = __builtin_bit_cast(two, v[0].x);
#pragma unroll
      for (int j = 0; j < LD; ++j) {
        most = __builtin_elementwise_max(most, __builtin_elementwise_max(__builtin_bit_cast(two, v[j].x), __builtin_bit_cast(two, v[j].y)));
        most = __builtin_elementwise_max(most, __builtin_elementwise_max(__builtin_bit_cast(two, v[j].z), __builtin_bit_cast(two, v[j].w)));
      }
      const int larger = max((int)most.x, (int)most.y);
      top = __uint_as_float((unsigned)larger << 16);
      exact = __any((unsigned)larger > 0x7F80u);
    }
    if (exact) {
      top = -INFINITY;
#pragma unroll
      for (int j = 0; j < LD; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) top = fmaxf(top, P::get(v[j], e));
    }
    lane_top = fmaxf(lane_top, top);
    bool by_table = false;
    if constexpr (TABLE) {
      by_table = __any(top >= -20.0f) && !__any(top >= 64.0f);
      if (by_table) {
#pragma unroll
        for (int j = 0; j < LD; ++j) asm volatile("" : "+v"(v[j].x), "+v"(v[j].y), "+v"(v[j].z), "+v"(v[j].w));  // (held as they are, not unpacked)
#pragma unroll
        for (int j = 0; j < LD; ++j) plain += Table::sum(table, v[j]);
      }
    }
    if (!by_table) {
      const float m_new = fmaxf(m, wave_max(top));
      if (m_new > -INFINITY && m_new < INFINITY) {
        if (m_new > m) s = m > -INFINITY ? s * exp_from(m, m_new) : 0.0;
        auto add = [&](auto log2) __attribute__((always_inline)) {
#pragma unroll
          for (int j = 0; j < LD; ++j) {
            double t[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) t[e] = log2(P::get(v[j], e));
            s += exp2_sum(t);
          }
        };
        if (fabsf(m_new) <= kNear) {
          const FromNear near(m_new);
          add([&](float x) { return near.log2(x); });
        } else {
          add([&](float x) { return log2_from((double)x, (double)m_new); });
        }
      }
      m = m_new;
    }
  }
  // ---- the sum ----
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    s += __shfl_xor(s, o);
    if (TABLE) plain += __shfl_xor(plain, o);
  }
  if (TABLE && plain > 0.0 && m < INFINITY) {  // both by one reference
    const float to = fmaxf(m, 0.0f);
    s = (m > -INFINITY ? s * exp_from(m, to) : 0.0) + plain * exp_from(0.0, to);
    m = to;
  }
  if (lane == 0) {
    sum_s[wv] = s;
    top_s[wv] = m;
  }
  // ---- the bound: by groups of a lane of every wavefront (groups of neighbours leave none where a run has few logits: 43 rows of 407 with
  // K = 17, bf16: 24 us with the merge, so 14) ----
  group_s[wv][lane] = lane_top;
  __syncthreads();
  if (wv == 0) {
    float mine = lane_top;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mine = fmaxf(mine, group_s[w][lane]);
    const unsigned place = (ordered(mine) & ~63u) | lane;  // (but for the last six bits, the lane's in the order)
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < 64; ++i) rank += (unsigned)__builtin_amdgcn_readlane(place, i) > place;
    if (rank == a.K - 1) bound_s = max(place & ~63u, ordered(-INFINITY) + 1);  // (-inf is no candidate)
  } else if (tid == 64) {
    float top = top_s[0];
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, top_s[w]);
    double sum = 0.0;
    for (int w = 0; w < kWaves; ++w)
      if (top_s[w] > -INFINITY && top < INFINITY) sum += sum_s[w] * exp_from(top_s[w], top);
    a.stats[blockIdx.x] = make_double2((double)top, sum);
  }
  __syncthreads();
  const float bound = logit_of(bound_s);
  if (lane_top >= bound) lane_s[atomicAdd(&count_s[0], 1)] = (unsigned short)tid;
  __syncthreads();
  // ---- the logits that reach it ----
  u64 *found = held[0];
  {
    const int pieces = end > begin ? (int)((end - begin + kWaves * (long)SUB - 1) / (kWaves * (long)SUB)) : 0, loads = pieces * LD, all = count_s[0] * loads;
    for (int i = tid; i < all && count_s[1] <= FOUND; i += THREADS) {
      const int l = (unsigned)i / (unsigned)loads, q = i - l * loads, from = lane_s[l];
      const long to = begin + ((long)(from >> 6) + (long)kWaves * (q / LD)) * SUB + ((q % LD) * 64 + (from & 63)) * VEC;
      if (to >= end) continue;
      const uint4 w = get(to);
      unsigned some = 0;
#pragma unroll
      for (int e = 0; e < VEC; ++e) some |= P::get(w, e) >= bound ? 1u << e : 0u;
      for (; some; some &= some - 1) {
        const int e = __builtin_ctz(some), k = atomicAdd(&count_s[1], 1);
        if (k < FOUND) found[k] = key_of(P::get(w, e), (int)(to + e));
      }
    }
  }
  __syncthreads();
  int n = count_s[1];
  if (n > FOUND) {  // (logits that are equal, or large ones in few lanes' places): every wavefront through its pieces, with a bound that rises
    u64 *mine = held[wv], least = (u64)bound_s << 32;
    __syncthreads();
    n = 0;
#pragma unroll 1
    for (at = begin + wv * SUB; at < end; at += kWaves * SUB)
#pragma unroll 1
      for (int j = 0; j < LD; ++j) {
        const long i = at + (j * 64 + lane) * VEC;
        const uint4 w = get(i);
        unsigned some = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) some |= P::get(w, e) >= logit_of((unsigned)(least >> 32)) ? 1u << e : 0u;
        while (__any(some != 0)) {
          const int e = some ? __builtin_ctz(some) : 0;
          const u64 key = key_of(P::get(w, e), (int)(i + e));
          unsigned long long in = __ballot(some != 0 && key >= least);
          if (n + __builtin_popcountll(in) > kHold) {
            n = keep_best(mine, n, a.K, lane);
            if (n == a.K) least = max(least, mine[a.K - 1] + 1);
            in = __ballot(some != 0 && key >= least);
          }
          if (in >> lane & 1ull) mine[n + __builtin_amdgcn_mbcnt_hi((unsigned)(in >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)in, 0))] = key;
          n += __builtin_popcountll(in);
          some &= some - 1;
        }
      }
    n = keep_best(mine, n, a.K, lane);
    const u64 key = lane < n ? mine[lane] : 0;
    if (lane == 0) have_s[wv] = n;
    __syncthreads();
    int before_me = 0;
    n = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      before_me += w < wv ? have_s[w] : 0;
      n += have_s[w];
    }
    if (key) found[before_me + lane] = key;
    __syncthreads();
  }
  u64 *out = a.lists_of + (size_t)blockIdx.x * a.K;
  for (int i0 = 0; i0 < n; i0 += THREADS / 4) {  // four lanes a key
    const int i = i0 + (tid >> 2);
    const u64 mine = found[min(i, n - 1)];
    int r = 0;
#pragma unroll 4
    for (int j = tid & 3; j < n; j += 4) r += found[j] > mine;
    r += __shfl_xor(r, 1);
    r += __shfl_xor(r, 2);
    if (i < n && r < a.K && (tid & 3) == 0) out[r] = mine;
  }
  if (tid < a.K && tid >= n) out[tid] = 0;
}

// Of n candidates in LDS, how many are before the i-th: four lanes a candidate, i = tid / 4.
__device__ __forceinline__ int rank_of(const u64 *p, const u64 *k, const unsigned char *w, int n, int i, int tid)
{
  const int at = min(i, n - 1), my_w = w[at];
  const u64 my_p = p[at], my_k = k[at];
  int r = 0;
#pragma unroll 4
  for (int j = tid & 3; j < n; j += 4) r += before(p[j], w[j], k[j], my_p, my_w, my_k);
  r += __shfl_xor(r, 1);
  return r + __shfl_xor(r, 2);
}

// log sum exp of W beams' rows from the `lists` sums of each: as many lanes a beam as it has sums.  It is left as the largest logit and the log of
// the sum by it: their own sum would lose of the log what the largest logit's unit is.
template <int THREADS>
__device__ __forceinline__ void join_sums(const double2 *stats, int W, int lists, int wv, int lane, double2 *lse_s)
{
  int per = 1;
  while (per < lists && per < 64) per *= 2;
  for (int w0 = wv * (64 / per); w0 < W; w0 += THREADS / per) {
    const int w = w0 + lane / per, at = lane % per;
    const double2 *st = stats + min(w, W - 1) * lists;
    double m = -INFINITY, s = 0.0;
    for (int i = at; i < lists; i += per) {
      const double2 x = st[i];
      if (!(x.x > -INFINITY)) continue;
      const double top = fmax(m, x.x);
      s = (m > -INFINITY ? s * exp_from(m, top) : 0.0) + x.y * exp_from(x.x, top);
      m = top;
    }
    double top = m;
    for (int o = per / 2; o >= 1; o >>= 1) top = fmax(top, __shfl_xor(top, o));
    s = m > -INFINITY ? s * exp_from(m, top) : 0.0;
    for (int o = per / 2; o >= 1; o >>= 1) s += __shfl_xor(s, o);
    if (at == 0 && w < W) lse_s[w] = make_double2(top, top == INFINITY ? 0.0 : log(s));
  }
}

// A key of a beam's candidate as a place in the order (only: the beam's first, and what it goes on as if it has ended); none: 0.
__device__ __forceinline__ u64 place_of(double score, double2 lse, bool ended, bool only, int eos, u64 &key)
{
  double to;
  if (ended) {  // goes on in one way
    key = key_of(0.0f, eos);
    to = only ? score : -INFINITY;
  } else {
    to = key == 0 ? -INFINITY : score + (((double)logit_of((unsigned)(key >> 32)) - lse.x) - lse.y);
  }
  return to > -INFINITY ? ordered(to) : 0;  // (a NaN neither)
}

// The K-th best of 64 groups' best.  Groups are a lane's of all wavefronts, in which first, second, .. elements of many lists meet: then about
// as many candidates reach the bound as groups do (without: one beam, 32 lists of 32: 27 us, so 7.6).
// One wavefront finds it: of 16 on a CU, four to a SIMD, each would wait for the other three.
template <int WAVES>
__device__ __forceinline__ u64 bound_of(u64 top, int K, int wv, int lane, u64 (*group_s)[64])
{
  group_s[wv][lane] = top;
  __syncthreads();
  if (wv == 0) {
    u64 mine = top;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) mine = max(mine, group_s[w][lane]);
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < 64; ++i) {
      const u64 o = (u64)(unsigned)__builtin_amdgcn_readlane((int)(mine >> 32), i) << 32 | (unsigned)__builtin_amdgcn_readlane((int)mine, i);
      rank += o > mine || (o == mine && i < lane);
    }
    if (rank == K - 1) group_s[0][0] = mine;
  }
  __syncthreads();
  return max(group_s[0][0], 1ull);
}
// the same of 32 bits, but for the last six of these (which hold the lane's place in the order)
template <int WAVES>
__device__ __forceinline__ unsigned bound_of(unsigned top, int K, int wv, int lane, unsigned (*group_s)[64])
{
  group_s[wv][lane] = top;
  __syncthreads();
  if (wv == 0) {
    unsigned mine = top;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) mine = max(mine, group_s[w][lane]);
    mine = (mine & ~63u) | lane;
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < 64; ++i) rank += (unsigned)__builtin_amdgcn_readlane(mine, i) > mine;
    if (rank == K - 1) group_s[0][0] = mine & ~63u;
  }
  __syncthreads();
  return group_s[0][0];
}

// The K best of n candidates in LDS, in order, for history b.
template <int THREADS>
__device__ __forceinline__ void write_best(const Args &a, int b, const u64 *p_s, const u64 *k_s, const unsigned char *w_s, const unsigned char *ended_s,
                                           int n, int tid)
{
  const size_t out = (size_t)b * a.K;
  for (int i0 = 0; i0 < n; i0 += THREADS / 4) {
    const int i = i0 + (tid >> 2);
    const int r = rank_of(p_s, k_s, w_s, n, i, tid);
    if (i >= n || r >= a.K || (tid & 3)) continue;
    const int item = item_of(k_s[i]), w = w_s[i];
    a.parent[out + r] = b * a.W + w;
    a.token[out + r] = item;
    a.out_score[out + r] = (float)score_of(p_s[i]);
    if (a.out_ended) a.out_ended[out + r] = item == a.eos || ended_s[w];
  }
  for (int r = n + tid; r < a.K; r += THREADS) {
    a.parent[out + r] = a.token[out + r] = -1;
    a.out_score[out + r] = -INFINITY;
    if (a.out_ended) a.out_ended[out + r] = 0;
  }
}

// One history: candidates that reach the K-th best of 64 groups' best are put in order.  Candidates are all that the lists hold or, of more than
// four a thread, those of the K lists with the best first elements.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void merge_kernel(Args a)
{
  constexpr int FEW = 4, MOST = FEW * THREADS;  // candidates of a thread, and of all
  constexpr bool CHOOSE = MOST >= kMost * kMost;  // (fewer threads are for fewer candidates)
  static_assert(!CHOOSE || kLists <= THREADS, "");
  __shared__ double2 lse_s[kMost];
  __shared__ double score_s[kMost];
  __shared__ u64 p_s[MOST], k_s[MOST], group_s[THREADS / 64][64];
  __shared__ short chosen_s[kMost];
  __shared__ unsigned char w_s[MOST], ended_s[kMost];
  __shared__ int count_s;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
  const int L = a.W * a.lists;
  const size_t row0 = (size_t)b * a.W;
  const u64 *lists = a.lists_of + row0 * a.lists * a.K;
  const bool few = !CHOOSE || L * a.K <= MOST;
  // Candidate tid + i THREADS: each list is turned round by another number of places (see bound_of).
  auto pick = [&](int i) -> int {
    const unsigned c = tid + i * THREADS, K = a.K, l = c / K;
    return (int)(l * K + (c + l + (l * K >> 6)) % K); 
  };
  // (requested at once: candidates or first elements, sums, scores)
  u64 key[FEW];
  int from[FEW];
#pragma unroll
  for (int i = 0; i < FEW; ++i) {
    from[i] = few ? pick(i) : tid + i * THREADS;
    key[i] = from[i] < (few ? L * a.K : L) ? lists[few ? from[i] : (size_t)from[i] * a.K] : 0;
  }
  if (tid < a.W) {
    score_s[tid] = (double)a.score[row0 + tid];
    ended_s[tid] = a.ended ? a.ended[row0 + tid] : 0;
  }
  if (tid == 0) count_s = 0;
  join_sums<THREADS>(a.stats + row0 * a.lists, a.W, a.lists, wv, lane, lse_s);
  __syncthreads();
  auto place = [&](int w, bool only, u64 &key) { return place_of(score_s[w], lse_s[w], ended_s[w], only, a.eos, key); };
  auto put = [&](u64 p, u64 k, int w) __attribute__((always_inline)) {
    const int to = atomicAdd(&count_s, 1);
    p_s[to] = p; k_s[to] = k; w_s[to] = (unsigned char)w;
  };
  int n_lists = 0;
  if constexpr (CHOOSE) {
    if (!few) {
      const int w = min((unsigned)tid / (unsigned)a.lists, (unsigned)a.W - 1);
      const u64 p = tid < L ? place(w, tid == w * a.lists, key[0]) : 0;
      const u64 bound = bound_of<THREADS / 64>(p, a.K, wv, lane, group_s);
      if (tid < L) {
        if (p >= bound) {
          const int to = atomicAdd(&count_s, 1);
          p_s[to] = p; k_s[to] = key[0]; w_s[to] = (unsigned char)w;
          // (which list it is: where the places of the last candidates will be)
          reinterpret_cast<int *>(p_s + MOST - kLists / 2)[to] = tid;
        }
      }
      __syncthreads();
      const int n = count_s;
      for (int i0 = 0; i0 < n; i0 += THREADS / 4) {
        const int i = i0 + (tid >> 2), r = rank_of(p_s, k_s, w_s, n, i, tid);
        if (i < n && r < a.K && (tid & 3) == 0) chosen_s[r] = (short)reinterpret_cast<int *>(p_s + MOST - kLists / 2)[i];
      }
      n_lists = min(n, a.K);
      __syncthreads();
      if (tid == 0) count_s = 0;
    }
  }
  // ---- the candidates ----
  u64 top = 0, at[FEW];
#pragma unroll
  for (int i = 0; i < FEW; ++i) {
    at[i] = 0;
    if (!few) from[i] = pick(i);
    const int c = from[i];
    if (few) {
      if (c >= L * a.K) continue;
      const int w = (unsigned)c / (unsigned)(a.lists * a.K);
      at[i] = place(w, c == w * a.lists * a.K, key[i]);
    } else {
      if (c >= n_lists * a.K) continue;
      const int r = (unsigned)c / (unsigned)a.K, j = c - r * a.K, l = chosen_s[r], w = (unsigned)l / (unsigned)a.lists;
      key[i] = r + j < a.K ? lists[(size_t)l * a.K + j] : 0;  // (r + j are before it)
      at[i] = r + j < a.K ? place(w, j == 0 && l == w * a.lists, key[i]) : 0;
    }
    top = max(top, at[i]);
  }
  const u64 bound = bound_of<THREADS / 64>(top, a.K, wv, lane, group_s);
#pragma unroll
  for (int i = 0; i < FEW; ++i) {
    const int c = from[i];
    if (at[i] >= bound) put(at[i], key[i], few ? (unsigned)c / (unsigned)(a.lists * a.K) : (unsigned)chosen_s[(unsigned)c / (unsigned)a.K] / (unsigned)a.lists);
  }
  __syncthreads();
  write_best<THREADS>(a, b, p_s, k_s, w_s, ended_s, count_s, tid);
}

// One history of few logits by itself: all of them are candidates, FEW a thread.
// Which candidates count is decided in 32 bits, with the bound on what these can be off by on the safe side; the few that may are put in order in
// 64.  A score in 32 bits is logit + c, c the beam's score less its sum: off by 2^-24 of c, of itself and of its sum with the bound, so by less than 2^-22
// (|c| + |logit|); the score in 64 bits, by less than 2^-48 of what c and the logit are differences of.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void few_kernel(Args a)
{
  constexpr int FEW = kFewLogits / 1024, MOST = FEW * THREADS, WAVES = THREADS / 64, N = 4;
  __shared__ u64 p_s[MOST], k_s[MOST];
  __shared__ unsigned group_s[WAVES][64];
  __shared__ double2 stats_s[kMost + WAVES], lse_s[kMost];
  __shared__ double score_s[kMost];
  __shared__ float2 off_s[kMost];
  __shared__ unsigned char w_s[MOST], ended_s[kMost];
  __shared__ int count_s;
  float *x_s = reinterpret_cast<float *>(p_s);  // (until candidates are put there)
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x, all = a.W * a.V;
  const size_t row0 = (size_t)b * a.W;
  const float by_V = 1.0f / (float)a.V;
  float x[FEW];
  int of[FEW];
#pragma unroll
  for (int i = 0; i < FEW; ++i) {
    const int c = tid + i * THREADS;
    of[i] = (int)(((float)c + 0.5f) * by_V);  // c / V: at least 1/2V from a whole number, and off by 64 * 2^-22
    x[i] = -INFINITY;
    if (c < all) {
      const int64_t at = (int64_t)(row0 + of[i]) * a.stride + (c - of[i] * a.V);
      x[i] = a.dtype == 0 ? element(static_cast<const float *>(a.logits) + at) : element(static_cast<const bf16_t *>(a.logits) + at);
    }
  }
  if (tid < a.W) {
    score_s[tid] = (double)a.score[row0 + tid];
    ended_s[tid] = a.ended ? a.ended[row0 + tid] : 0;
  }
  if (tid == 0) count_s = 0;
#pragma unroll
  for (int i = 0; i < FEW; ++i) x_s[tid + i * THREADS] = x[i];
  __syncthreads();
  // ---- the rows' sums: as many threads a row as there are for each, a power of two; up to 64 sum among themselves ----
  const int each_log2 = 31 - __builtin_clz(THREADS / a.W), lanes = min(1 << each_log2, 64), parts = (1 << each_log2) / lanes;
  {
    const int q = tid / lanes, w = q / parts, each = (a.V + parts - 1) / parts, from = (q - w * parts) * each;
    const int n = w < a.W ? min(each, a.V - from) : 0, i0 = tid % lanes;
    const float *row = x_s + w * a.V + from;
    float m = -INFINITY;
    for (int i = i0; i < n; i += lanes) m = fmaxf(m, row[i]);  // (a NaN is ruled out: fmaxf takes the other)
    for (int o = lanes / 2; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    double s = 0.0;
    if (m > -INFINITY && m < INFINITY) {
      for (int i = i0; i < n; i += lanes * N) {
        double t[N];
#pragma unroll
        for (int j = 0; j < N; ++j) t[j] = log2_from(i + lanes * j < n ? (double)row[i + lanes * j] : -INFINITY, (double)m);
        s += exp2_sum(t);
      }
    }
    for (int o = lanes / 2; o >= 1; o >>= 1) s += __shfl_xor(s, o);
    if (i0 == 0 && w < a.W) stats_s[q] = make_double2((double)m, s);
  }
  __syncthreads();
  join_sums<THREADS>(stats_s, a.W, parts, wv, lane, lse_s);
  __syncthreads();
  // ---- the candidates ----
  if (tid < a.W) {
    const double c = (score_s[tid] - lse_s[tid].x) - lse_s[tid].y;
    const float by_64 = fmaf(0x1p-48f, fabsf((float)score_s[tid]) + fabsf((float)lse_s[tid].x), 0x1p-120f);
    // (ended, or beyond 32 bits: each is a candidate, and none bounds the others.  -inf or NaN: none is a candidate)
    off_s[tid] = ended_s[tid] || fabs(c) > 1e30 ? make_float2(0.0f, INFINITY) : make_float2((float)c, fmaf(0x1p-22f, fabsf((float)c), by_64));
    if (!ended_s[tid] && !(c > -INFINITY)) off_s[tid] = make_float2(-INFINITY, 0.0f);
  }
  __syncthreads();
  float upto[FEW], least = -INFINITY;
#pragma unroll
  for (int i = 0; i < FEW; ++i) {
    const int c = tid + i * THREADS, w = min(of[i], a.W - 1);
    const float2 off = off_s[w];
    const float near = x[i] + off.x, by = fmaf(fabsf(x[i]), 0x1p-22f, off.y);
    const bool is = c < all && off.x > -INFINITY && (ended_s[w] ? c == w * a.V : x[i] > -INFINITY);
    upto[i] = is ? near + by : -INFINITY;
    if (is && by < INFINITY) least = fmaxf(least, near - by);
    if (is && !(by < INFINITY)) upto[i] = INFINITY;
  }
  const float reach = logit_of(max(bound_of<WAVES>(ordered(least), a.K, wv, lane, group_s), ordered(-INFINITY)));
#pragma unroll
  for (int i = 0; i < FEW; ++i) {
    if (!(upto[i] > -INFINITY && upto[i] >= reach)) continue;
    const int c = tid + i * THREADS, w = of[i], item = c - w * a.V;
    u64 key = key_of(x[i], item);
    const u64 p = place_of(score_s[w], lse_s[w], ended_s[w], item == 0, a.eos, key);
    if (p == 0) continue;
    const int to = atomicAdd(&count_s, 1);
    p_s[to] = p; k_s[to] = key; w_s[to] = (unsigned char)w;
  }
  __syncthreads();
  write_best<THREADS>(a, b, p_s, k_s, w_s, ended_s, count_s, tid);
}

namespace {

long piece(int dtype, int loads) { return 64l * loads * (dtype == 0 ? 4 : 8); }

}  // namespace

void plan(Args &a)
{
  // A history of up to 8192 logits is one workgroup's, but where these are large ones in several rounds for few beams each, which rows by
  // themselves fill better (4 beams of 1682 logits: 10.5 us, in two kernels 11.3; 160 histories of 26 beams of 42: 9.5, 47; 250 of 4 of 2000:
  // 11.5, 14.8; 1000: 41, 33; 1000 of one beam of 8000: 48, 23; 300 of 32 of 256: 24, 97).
  a.lists = 0;
  const long logits = (long)a.W * a.V;
  if (logits <= kFewLogits / 4 || (logits <= kFewLogits && (a.B <= 256 || a.W > 5))) return;
  // Runs: a workgroup for each of the CUs' two places, or as comes near (2048, 1024 and 512 workgroups for 512 rows of 152063: 52, 49 and 39
  // us; 508 and 762 for 254 rows of 108488: 26 and 30 with the merge); no more than the merge's small workgroup takes, unless runs become long (8 rows of 150001, K = 8: merge 6 us with 16 lists a row, 10 with 37).
  // Four loads a lane and piece of bf16, two of fp32 (400000 logits, K = 32: 9 us, four 23, one 10; 512 rows of 152063: 85, 84, 99); one in
  // short runs: then a lane's few logits are not worth a table either (1024 rows of 5000: 13 us for 19).
  const long rows = (long)a.B * a.W, small = kWaves * piece(a.dtype, 1), large = kWaves * piece(a.dtype, 4);
  const long light = a.W * a.K <= kFewCandidates ? kFewCandidates / (a.W * a.K) : 1;
  long lists = 1, most = a.V <= 8 * large * light ? light : kLists / a.W;
  if (most > (a.V + small - 1) / small) most = (a.V + small - 1) / small;
  // (a round of 512 workgroups takes as long as its logits and 30000 more)
  for (long n = 2, best = 0; n <= most && (n - 1) * rows < 1024; ++n) {
    const auto cost = [&](long of) { return (of * rows + 511) / 512 * ((a.V + of - 1) / of + 30000); };
    if (!best) best = cost(1);
    if (cost(n) < best) best = cost(n), lists = n;
  }
  a.loads = (a.V + lists - 1) / lists <= 3 * small ? 1 : a.dtype == 0 ? 2 : 4;
  const long pieces = (a.V + piece(a.dtype, a.loads) - 1) / piece(a.dtype, a.loads);
  a.subs = (int)((pieces + lists - 1) / lists);
  a.lists = (int)((pieces + a.subs - 1) / a.subs);
}

bool launch(const Args &a, hipStream_t st)
{
  if (a.lists == 0) {
    const bool small = a.W * a.V <= kFewLogits / 4;
    if ((long)a.B * (small ? 256 : 1024) >= 1l << 32) return false;
    if (small) hipLaunchKernelGGL((few_kernel<256>), dim3((unsigned)a.B), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((few_kernel<1024>), dim3((unsigned)a.B), dim3(1024), 0, st, a);
    return true;
  }
  const long blocks = (long)a.B * a.W * a.lists;
  if (blocks * 64 * kWaves >= 1l << 32) return false;
  [&] {
    auto rows = [&](auto kernel) { BLOSSOM_LAUNCH(kernel, dim3((unsigned)blocks), dim3(64 * kWaves), 0, st, a); };
    if (a.dtype == 0 && a.loads > 1) rows(rows_kernel<float, 2, false>);
    else if (a.dtype == 0) rows(rows_kernel<float, 1, false>);
    else if (a.loads > 1) rows(rows_kernel<bf16_t, 4, true>);
    else rows(rows_kernel<bf16_t, 1, false>);
    if (launch_failed()) return;
    if (a.W * a.lists * a.K <= kFewCandidates) BLOSSOM_LAUNCH((merge_kernel<256>), dim3((unsigned)a.B), dim3(256), 0, st, a);
    else BLOSSOM_LAUNCH((merge_kernel<1024>), dim3((unsigned)a.B), dim3(1024), 0, st, a);
  }();
  return true;
}

}  // namespace beam
}  // namespace blossom
