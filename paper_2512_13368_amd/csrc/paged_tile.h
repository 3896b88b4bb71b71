// Key tiles of a paged cache in LDS: 32 rows of K or V, moved from their pages by direct global->LDS loads, and the operands that
// 16x16 matrix instructions take from them (gfx950 only).
//
// A load moves 1 KB, lane l's 16 bytes to 16*l from its destination on: neighbouring lanes take neighbouring bytes of a row, at 64
// bytes a clock and CU.  (A lane a row, as the matrix instructions want their operands, gets 18 bytes a clock: the rows of
// neighbouring lanes are fetched one at a time.)
#pragma once

#include "common.h"
#include "mfma_common.h"
#include "paged.h"

namespace blossom {
namespace paged {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kTile = 32;  // keys

// what stands in for rows that nobody may see
static __device__ const uint4 kZeros[64] = {};

// 16 bytes a lane to `lds` + 16 * lane: from a uniform base and 32-bit offsets, or from an address a lane.  ONCE: past the caches.
template <bool ONCE>
__device__ __forceinline__ void to_lds(const void *base, unsigned off, unsigned lds)
{
  if constexpr (ONCE) asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"{m0}"(lds), "v"(off), "s"(base) : "memory");
  else asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(lds), "v"(off), "s"(base) : "memory");
}
template <bool ONCE>
__device__ __forceinline__ void to_lds(const void *from, unsigned lds)
{
  if constexpr (ONCE) asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"{m0}"(lds), "v"(from) : "memory");
  else asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(lds), "v"(from) : "memory");
}
// at most N of this wavefront's requests are still on their way
template <int N>
__device__ __forceinline__ void arrived()
{
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <typename T, int D>
struct Tile {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int RB = D * (int)sizeof(T);            // bytes of a row
  static constexpr int CH = RB / 16;                       // 16-byte chunks of a row
  static constexpr int RPL = 64 / CH;                      // rows that a load moves
  static constexpr int LOADS = RPL < kTile ? kTile / RPL : 1;
  static constexpr int BYTES = LOADS * 1024;               // of LDS (rows of 16 bytes: the second half is not used)
  static constexpr int NK = BF ? (D >= 32 ? D / 32 : 1) : (D >= 16 ? D / 16 : 1);  // 16-byte pieces of a lane's query and key rows
  static constexpr int NV = D >= 16 ? D / 16 : 1;          // accumulators: 16 channels each

  // LDS position of chunk c of row r: c ^ swz(r).  The 16 lanes that one clock of a 16-byte read serves (0-3, 12-15 of one lane
  // group, 4-11 of the next), or the 32 of an 8-byte one, then meet every bank once.
  static __device__ __forceinline__ int swz_k(int r)
  {
    if (RB >= 256) return r & 15;
    if (RB == 128) return (r >> 1) & 7;
    if (RB == 64) return (0x78 >> (2 * ((r >> 2) & 3))) & 3;
    return 0;
  }
  static __device__ __forceinline__ int swz_v(int r)
  {
    if (!BF) return RB == 512 ? (r >> 2) & 1 : 0;
    if (RB == 256) return 2 * (r & 7);
    if (RB == 128) return 2 * ((r >> 1) & 3);
    if (RB == 64) return 2 * ((r >> 2) & 1);
    return 0;
  }

  // Requests loads first, first + step, .. of a tile's K and V.  Lane l < 32 knows where row l of the tile lies (`off`, bytes from
  // either cache's beginning) and whether it is anybody's (`ok`); `whole`: all are.
  template <bool ONCE>
  static __device__ __forceinline__ void request(const Args &a, const char *ks, const char *vs, size_t off, bool ok, bool whole, int lane,
                                                 int first, int step)
  {
    const char *Kc = static_cast<const char *>(a.K_cache), *Vc = static_cast<const char *>(a.V_cache);
    const unsigned k_to = mfma::lds_address(ks), v_to = mfma::lds_address(vs);
    const int l_row = lane / CH, l_pos = lane % CH;
    const unsigned lo = (unsigned)off, hi = (unsigned)(off >> 32);
    if (RPL <= 8 && whole) {  // (rows that start at a multiple of RPL lie in one page, one after another)
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        if (step > 1 && i % step != first) continue;
        const int r = RPL * i + l_row;
        const size_t base = (size_t)(unsigned)__builtin_amdgcn_readlane(hi, RPL * i & 31) << 32 | (unsigned)__builtin_amdgcn_readlane(lo, RPL * i & 31);
        to_lds<ONCE>(Kc + base, l_row * RB + (l_pos ^ swz_k(r)) * 16, k_to + i * 1024);
        to_lds<ONCE>(Vc + base, l_row * RB + (l_pos ^ swz_v(r)) * 16, v_to + i * 1024);
      }
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        if (step > 1 && i % step != first) continue;
        const int r = min(RPL * i + l_row, kTile - 1);
        const size_t mine = (size_t)(unsigned)__shfl((int)hi, r) << 32 | (unsigned)__shfl((int)lo, r);
        const bool there = __shfl((int)ok, r) != 0;
        to_lds<ONCE>(there ? Kc + mine + (l_pos ^ swz_k(r)) * 16 : reinterpret_cast<const char *>(kZeros), k_to + i * 1024);
        to_lds<ONCE>(there ? Vc + mine + (l_pos ^ swz_v(r)) * 16 : reinterpret_cast<const char *>(kZeros), v_to + i * 1024);
      }
    }
  }

  // A row of Q as an operand: lane group c's pieces.  Channels beyond the row are zeros.
  struct Query {
    uint4 x[NK];
  };
  static __device__ __forceinline__ void load_query(Query &q, const T *p, int c)
  {
#pragma unroll
    for (int i = 0; i < NK; ++i)
      q.x[i] = (4 * i + c) * 16 < RB ? *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p) + (4 * i + c) * 16) : make_uint4(0, 0, 0, 0);
  }

  // Logits of keys 16h .. 16h + 15 (matrix rows) with a lane's query (column n): lane group c gets those of keys 16h + 4c + i.
  static __device__ __forceinline__ f32x4 logits(const char *ks, int h, int n, int c, const Query &q)
  {
    const int r = 16 * h + n;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      uint4 k = make_uint4(0, 0, 0, 0);
      if (CH >= 4 || c < CH) k = *reinterpret_cast<const uint4 *>(ks + r * RB + (((4 * i + c) ^ swz_k(r)) * 16));
      if constexpr (BF) {
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(mfma::bf16x8, k), __builtin_bit_cast(mfma::bf16x8, q.x[i]), s, 0, 0, 0);
      } else {
        const f32x4 kf = __builtin_bit_cast(f32x4, k), qf = __builtin_bit_cast(f32x4, q.x[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[e], s, 0, 0, 0);
      }
    }
    return s;
  }

  // acc += V^T P^T: p[4h + i] is the probability of key 16h + 4c + i.  The sum over keys may run in any order, so lane group c takes
  // the keys whose probabilities it holds.  bf16: V^T comes through the transposing LDS read, P is rounded as the matrix instruction wants
  // it (its sum is of the unrounded ones).  FINE: what that leaves of P goes through a second product with the same V, so that of the
  // output's error its own rounding is all there is (1.6e-3 of its norm; with P rounded once 2.0 to 2.4e-3).  Memory-bound kernels have
  // the time: 100 to 1024 keys at d = 64 15.1 us without and 15.4 with, 131071 at d = 128 85.6 and 86.0, 16 chosen pages 8.1 and 8.5.
  // Accumulator j, element i holds channel channel(j, c, i) of the lane's query.  `both`: the tile's second 16 keys count too.
  template <bool FINE>
  static __device__ __forceinline__ void product(const char *vs, const float (&p)[8], bool both, int lane, f32x4 (&acc)[NV])
  {
    const int n = lane & 15, c = lane >> 4;
    if constexpr (BF) {
      mfma::bf16x8 pf, rest;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        pf[i] = (__bf16)p[i];
        if constexpr (FINE) rest[i] = (__bf16)(p[i] - (float)pf[i]);
      }
      const int r = 4 * c + (n >> 2);  // (and 16 on: the same swizzle)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int ch = CH >= 2 ? 2 * j + ((n >> 1) & 1) : 0;
        const char *v = vs + r * RB + ((ch ^ swz_v(r)) * 16) + (n & 1) * 8;
        const mfma::s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mfma::lds_s16x4 *)(v));
        const mfma::s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mfma::lds_s16x4 *)(v + 16 * RB));
        const mfma::bf16x8 vt = __builtin_bit_cast(mfma::bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        if constexpr (FINE) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, rest, acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pf, acc[j], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        if (s == 4 && !both) break;
        const int r = 16 * (s >> 2) + 4 * c + (s & 3);
        const char *row = vs + r * RB;
        float v[NV];
        if constexpr (NV >= 4) {
#pragma unroll
          for (int e = 0; e < NV; e += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(row + (((NV * n + e) / 4) ^ swz_v(r)) * 16);
            v[e] = x.x; v[e + 1] = x.y; v[e + 2] = x.z; v[e + 3] = x.w;
          }
        } else if constexpr (NV == 2) {
          const float2 x = *reinterpret_cast<const float2 *>(row + n * 8);
          v[0] = x.x; v[1] = x.y;
        } else {
          v[0] = *reinterpret_cast<const float *>(row + (D == 8 ? n & 7 : n) * 4);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j], p[s], acc[j], 0, 0, 0);
      }
    }
  }
  // (d = 8: channels 8 .. 15 repeat 0 .. 7 and are dropped)
  static __device__ __forceinline__ int channel(int j, int c, int i) { return BF ? 16 * j + 4 * c + i : NV * (4 * c + i) + j; }
};

__device__ __forceinline__ void store_out(float *p, float x) { *p = x; }
__device__ __forceinline__ void store_out(bf16_t *p, float x) { p->bits = __builtin_bit_cast(uint16_t, (__bf16)x); }

__device__ __forceinline__ void store_four(float *p, const float4 &x, float f)
{
  *reinterpret_cast<float4 *>(p) = make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
}
__device__ __forceinline__ void store_four(bf16_t *p, const float4 &x, float f)
{
  *reinterpret_cast<uint2 *>(p) = make_uint2(mfma::pack2_bf16(x.x * f, x.y * f), mfma::pack2_bf16(x.z * f, x.w * f));
}

// Maximum over the four lanes that hold a row's logits.
__device__ __forceinline__ float row_max(float x)
{
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const u32x2 b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// A wavefront's 16 rows over the tiles it has met: reference (log2 units) and sum in fp32, unnormalised output.  The reference is a
// row's maximum over the first keys it met; it is raised only when a lane's eight probabilities of a tile pass kSumLimit in sum, so the
// usual tile takes no maximum; where it is far from 0 (see kFar), a tile takes one and has its logits scaled before it is subtracted.
constexpr float kSumLimit = 4096.0f;
template <typename T, int D>
struct Rows {
  typedef Tile<T, D> TL;
  f32x4 acc[TL::NV];
  float m, l;  // (l: this lane's keys alone; m is -inf while the row has met no key)
  // (a row that is nobody's, `on` false, never meets one and need not be waited for)
  __device__ __forceinline__ void clear(bool on = true)
  {
    m = on ? mfma::kNegInf : 0.0f;
    l = 0.0f;
#pragma unroll
    for (int j = 0; j < TL::NV; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // one tile; bit k of `seen`: this lane's row sees key k of the tile (all: no key is masked for any row; both: any row sees one of
  // the second 16)
  template <bool FINE>
  __device__ __forceinline__ void attend(const char *ks, const char *vs, const typename TL::Query &q, float scale2, unsigned seen, bool all, bool both,
                                         int lane)
  {
    const int n = lane & 15, c = lane >> 4;
    float s[8], p[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 0 || both) {
        const f32x4 x = TL::logits(ks, h, n, c, q);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * h + i] = x[i];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * h + i] = mfma::kNegInf;
      }
    }
    if (!all) {
      const int mine = (int)(seen >> (4 * c));
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * h + i] = mine >> (16 * h + i) & 1 ? s[4 * h + i] : mfma::kNegInf;
    }
    bool place = __any(is_far(m));  // (-inf too)
    float sum, scale = scale2;
#pragma unroll 1
    for (;;) {
      float ref = m;
      if (place) {
        const float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
        const float to = fmaxf(m, row_max(mx) * scale2);
        ref = to == mfma::kNegInf ? 0.0f : to;  // no key seen yet: every exponential is 0
        const float f = __builtin_amdgcn_exp2f(m - ref);
        m = to;
        l *= f;
#pragma unroll
        for (int j = 0; j < TL::NV; ++j) acc[j] *= f;
        if (__any(is_far(ref))) {
#pragma unroll
          for (int i = 0; i < 8; ++i) s[i] = rounded_product(s[i], scale2);
          scale = 1.0f;
        }
      }
      sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale, -ref));
        sum += p[i];
      }
      if (place || !__any(!(sum <= kSumLimit))) break;
      place = true;
    }
    l += sum;
    TL::template product<FINE>(vs, p, both, lane, acc);
  }
  __device__ __forceinline__ float total() const
  {
    float x = l + __shfl_xor(l, 16);
    return x + __shfl_xor(x, 32);
  }
};

}  // namespace paged
}  // namespace blossom
