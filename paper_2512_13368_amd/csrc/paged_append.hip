// New tokens' keys and values into a paged cache, with the rotary position embedding on the way (Sec. 3.3), Q rotated too.
//
// A wavefront takes one token, or a share of its rows where there are few tokens: rows of Q, K and V are d elements each, a lane
// moves 16 bytes, and a lane's place inside a row is the same in every row it moves, so that the token's angles are read once.
// Nothing is read twice and nothing needs LDS: the kernel is bound by memory (16383 tokens of 32 + 2 * 8 heads of 128 bf16 channels,
// 411 MB in and out: 73 us, 5.6 TB/s, where a copy of 1 GiB reaches 6.2), one token a sequence by the launch and the chain of loads
// from a token to its page (128 sequences: 4.5 us).
#include "common.h"
#include "launch.h"
#include "paged.h"

namespace blossom {
namespace paged {

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;  // loads of a lane on their way together

// 16 bytes; ONCE: past the caches
template <bool ONCE>
__device__ __forceinline__ uint4 get(const uint4 *p)
{
  if constexpr (ONCE) return load_once(p);
  else return *p;
}
template <bool ONCE>
__device__ __forceinline__ void put(uint4 *p, const uint4 &v)
{
  typedef unsigned words __attribute__((ext_vector_type(4)));
  if constexpr (ONCE) __builtin_nontemporal_store(__builtin_bit_cast(words, v), reinterpret_cast<words *>(p));
  else *p = v;
}


// 16 bytes of a row, as floats
template <typename T>
struct Chunk;
template <>
struct Chunk<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ void get(const uint4 &v, float (&x)[4])
  {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&x)[4])
  {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <>
struct Chunk<bf16_t> {
  static constexpr int E = 8;
  static __device__ __forceinline__ void get(const uint4 &v, float (&x)[8])
  {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  // (round to nearest even by the hardware's conversion, which keeps NaN a NaN)
  static __device__ __forceinline__ uint4 put(const float (&x)[8])
  {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const pair p = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
      w[i] = __builtin_bit_cast(uint32_t, p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

}  // namespace

// `share`: wavefronts that divide a token's rows (a power of two).  TREE: drafted tokens, which are turned by their places in their trees.
template <typename T, bool ONCE, bool TREE>
__global__ __launch_bounds__(kThreads) void append_kernel(Args a, int share)
{
  constexpr int E = Chunk<T>::E;
  const int lane = threadIdx.x & 63;
  const long wave = (long)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = (int)(wave / share), part = (int)(wave % share);
  if (t >= a.T) return;
  const Sequence seq(a, lane, [&](int, int cu) { return cu <= t; });
  const int s = seq.s, lo = seq.first, hi = seq.first + seq.count;
  if (t < lo || t >= hi) return;  // a row that no sequence owns
  const int n = a.kv_len[s];
  const long pos = (long)n - (hi - lo) + (t - lo);
  long angle = pos;
  if constexpr (TREE) angle = (long)n - (hi - lo) + depth_of(a.tree[t], t - lo, hi - lo);
  const bool placed = pos >= 0 && pos < a.cap && (!TREE || (angle >= 0 && angle < a.cap));
  int id = -1;
  if (placed) id = a.page_table[s * a.table_seq + (pos >> a.page_shift)];
  const bool stored = id >= 0 && id < a.n_pages;
  const int page = 1 << a.page_shift, slot = (int)(pos & (page - 1));

  const int lanes = a.d / E;            // lanes of a row
  const int at = (lane % lanes) * E;    // this lane's channels in every row it moves
  float c[E / 2], sn[E / 2];
#pragma unroll
  for (int i = 0; i < E / 2; ++i) { c[i] = 1.0f; sn[i] = 0.0f; }
  if (a.rope_cos && placed) {
    const float *pc = a.rope_cos + angle * (a.d / 2) + at / 2, *ps = a.rope_sin + angle * (a.d / 2) + at / 2;
#pragma unroll
    for (int i = 0; i < E / 2; i += 2) {
      const float2 x = *reinterpret_cast<const float2 *>(pc + i), y = *reinterpret_cast<const float2 *>(ps + i);
      c[i] = x.x; c[i + 1] = x.y;
      sn[i] = y.x; sn[i + 1] = y.y;
    }
  }
  auto turn = [&](const uint4 &v) __attribute__((always_inline)) -> uint4 {
    float x[E];
    Chunk<T>::get(v, x);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {  // the recipe of the selection's rotation
      const float p = x[2 * i + 1] * sn[i], u = x[2 * i + 1] * c[i];
      x[2 * i + 1] = fmaf(x[2 * i], sn[i], u);
      x[2 * i] = fmaf(x[2 * i], c[i], -p);
    }
    return Chunk<T>::put(x);
  };

  const int per = 64 / lanes;  // rows that a wavefront moves at a time
  const int nq = a.Q ? a.H : 0, rows = nq + 2 * a.G;
  const T *Q = static_cast<const T *>(a.Q), *K = static_cast<const T *>(a.K), *V = static_cast<const T *>(a.V);
  T *Kc = static_cast<T *>(a.K_cache), *Vc = static_cast<T *>(a.V_cache), *Qr = static_cast<T *>(a.Q_rot);
  const size_t cell = (size_t)(stored ? id : 0) * a.G * page * a.d + (size_t)slot * a.d + at;
  // row r's chunk: where it is, where it goes (nullptr: nowhere)
  auto from = [&](int r) __attribute__((always_inline)) -> const uint4 * {
    const T *p = r < nq ? Q + t * a.q_stride + (size_t)r * a.d
                        : r < nq + a.G ? K + t * a.k_stride + (size_t)(r - nq) * a.d : V + t * a.v_stride + (size_t)(r - nq - a.G) * a.d;
    return reinterpret_cast<const uint4 *>(p + at);
  };
  auto to = [&](int r) __attribute__((always_inline)) -> uint4 * {
    T *p = r < nq ? Qr + ((size_t)t * a.H + r) * a.d + at : (r < nq + a.G ? Kc + (size_t)(r - nq) * page * a.d : Vc + (size_t)(r - nq - a.G) * page * a.d) + cell;
    return reinterpret_cast<uint4 *>(p);
  };
  const int first = part * per + lane / lanes, step = share * per;
  for (int r0 = first; r0 < rows; r0 += kBatch * step) {
    uint4 v[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int r = r0 + k * step;
      if (r < rows) v[k] = get<ONCE>(from(r));
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int r = r0 + k * step;
      if (r >= rows || (r >= nq && !stored)) continue;
      if (r < nq && !placed) v[k] = make_uint4(0, 0, 0, 0);
      else if (r < nq || (r < nq + a.G && a.rope_cos)) v[k] = turn(v[k]);
      put<ONCE>(to(r), v[k]);
    }
  }
}

bool launch_append(const Args &a, hipStream_t st)
{
  // few tokens: their rows go to more wavefronts, as far as a wavefront has a load's worth of rows left
  const int rows = (a.Q ? a.H : 0) + 2 * a.G, per = 64 * 16 / (a.d * (a.dtype == 0 ? 4 : 2));
  int share = 1;
  while ((long)a.T * share < 2048 && share * per < rows) share *= 2;
  const long waves = (long)a.T * share;
  const long blocks = (waves + kThreads / 64 - 1) / (kThreads / 64);
  if (!countable(blocks, kThreads)) return false;
  // More than half the last-level cache is written past it: 16383 tokens of 32 + 2 * 8 heads of 128 channels, 201 MB, take 73 us so and
  // 82 kept.  What is less stays for the attention that follows.
  const bool once = (double)a.T * rows * a.d * (a.dtype == 0 ? 4 : 2) > 128e6;
  auto go = [&](auto kernel) { BLOSSOM_LAUNCH(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, st, a, share); };
  auto pick = [&](auto tree) {
    constexpr bool TREE = decltype(tree)::value;
    if (a.dtype == 0 && once) go(append_kernel<float, true, TREE>);
    else if (a.dtype == 0) go(append_kernel<float, false, TREE>);
    else if (once) go(append_kernel<bf16_t, true, TREE>);
    else go(append_kernel<bf16_t, false, TREE>);
  };
  if (a.tree) pick(std::true_type{});
  else pick(std::false_type{});
  return true;
}

}  // namespace paged
}  // namespace blossom
