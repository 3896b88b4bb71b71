// The paged key/value cache's operators: kernel-side description and what their kernels share (gfx950 only).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "common.h"

namespace blossom {
namespace paged {

// Division of numbers below 2^31 by one divisor: floor(n m / 2^(31 + s)) with s = ceil(log2 d), m = ceil(2^(31 + s) / d), which is
// exact because n (m d - 2^(31 + s)) < 2^(31 + s).
struct Divisor {
  uint32_t m, s;
  __device__ __forceinline__ int of(int n) const { return (int)((uint64_t)(uint32_t)n * m >> (31 + s)); }
};
inline Divisor divisor(uint32_t d)
{
  uint32_t s = 0;
  while ((1ull << s) < d) ++s;
  return {(uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
}

// One call (passed to kernels by value; device pointers).  Element type of Q, K, V, the caches and O: `dtype`.
struct Args {
  int S, T, H, G, R, d;        // sequences, packed new tokens, heads, key/value heads, H / G, head size
  Divisor by_G, by_H, by_R, by_parts;
  int page_shift;              // log2 of the positions a page holds
  int n_pages, max_pages;      // pages of a cache, entries of a page-table row
  int cap;                     // positions a sequence may have: keys at or beyond are never read or written
  int window;                  // a query sees that many positions up to its own; 0x7FFFFFFF: all
  int dtype;
  float scale2;                // softmax scale * log2(e)
  int64_t table_seq, table_group;  // page-table steps from a sequence and from a key/value head to the next
  const void *Q, *K, *V;
  int64_t q_stride, k_stride, v_stride;  // elements from a token's row to the next's
  void *K_cache, *V_cache;     // [n_pages, G, page, d]
  const int *page_table, *cu, *kv_len;
  const float *rope_cos, *rope_sin;  // [cap, d/2] or nullptr
  void *Q_rot;                 // [T,H,d] or nullptr
  void *O;                     // [T,H,d] (decode: [S,H,d])
  float *lse;                  // [T,H] or nullptr
  int parts;                   // decode: workgroups that share a key/value head's keys (0: one a sequence); prompt: parts of a row's keys
  float *part_o, *part_ml;     // their sums [H, parts, d] and (reference in log2 units, sum of exponentials) [H, parts, 2], in the
                               // workspace; prompt: [T, H, parts, ..]
  int row_tiles;               // prompt: workgroups a key/value head and part
  int2 *part_of;               // decode: [S] first part and parts of a sequence, there too
};

// HIP counts a launch's threads in 32 bits.  The launchers below start nothing and return false for a call that would have more.
inline bool countable(long workgroups, int threads) { return workgroups * threads < 1l << 32; }

// append: paged_append.hip
bool launch_append(const Args &a, hipStream_t st);
// one-token and prompt attention: paged_attn.hip.  decode_parts, prompt_parts: what `parts` is for this shape
int decode_parts(const Args &a);
int prompt_parts(const Args &a);
bool launch_decode(const Args &a, hipStream_t st);
bool launch_prompt(const Args &a, hipStream_t st);
// prompt attention for bf16, d = 64 or 128: paged_prompt.hip
constexpr int kPromptRows = 128;  // query rows of a workgroup, which has four wavefronts
constexpr int kPromptWaves = 4;
bool prompt_mfma_supported(const Args &a);
void launch_prompt_mfma(const Args &a, hipStream_t st);
// prompt attention for everything else: paged_shared.hip
// rows of a workgroup: 16 a wavefront, of which there are as many as it takes to move a tile
constexpr int shared_waves(int row_bytes) { return row_bytes >= 256 ? 4 : 2; }
void launch_prompt_shared(const Args &a, hipStream_t st);

// Calls f with the element type and the head size as compile-time constants.
template <typename F>
inline void with_type(const Args &a, F &&f)
{
  auto with_dim = [&](auto type) {
    switch (a.d) {
      case 8: f(type, std::integral_constant<int, 8>{}); break;
      case 16: f(type, std::integral_constant<int, 16>{}); break;
      case 32: f(type, std::integral_constant<int, 32>{}); break;
      case 64: f(type, std::integral_constant<int, 64>{}); break;
      default: f(type, std::integral_constant<int, 128>{}); break;
    }
  };
  if (a.dtype == 0) with_dim(0.0f);
  else with_dim(bf16_t{});
}

// A probability is 2^(scale2 s - ref) with the product unrounded and the reference a rounded one, so the largest key's is 2^e, e the
// rounding of the reference: what numerator and denominator share and the log of the sum takes back.  Beyond kFar e may be anything
// (half a unit of a reference of 2^33 is 512), so the products of such rows' tiles are rounded like the reference.  That is no less
// exact than the logits themselves, and is done where it is needed alone: for a walk of usual logits it is a comparison a tile.
constexpr float kFar = 1048576.0f;
__device__ __forceinline__ bool is_far(float ref) { return fabsf(ref) > kFar; }
// x f in 32 bits, whatever becomes of it
__device__ __forceinline__ float rounded_product(float x, float f)
{
#pragma clang fp contract(off)
  return x * f;
}

// Keys lo .. hi that a query at `pos` sees, of a sequence with n keys (hi < lo: none).
struct Range {
  int lo, hi;
};
__device__ __forceinline__ Range seen_by(const Args &a, int pos, int n)
{
  if (pos < 0) return {0, -1};
  return {max(pos - a.window + 1, 0), min(pos, min(n, a.cap) - 1)};
}

// Rows that see fewer keys than this have large probabilities, whose rounding to bf16 would show beside outputs that are averages over
// many keys: workgroups that have such rows keep what it leaves (see FINE in paged_tile.h), in every kernel.
constexpr int kFewKeys = 32;
// Does any row between two of one sequence see so few?  (The number rises with the position, and falls beyond the capacity.)
__device__ __forceinline__ bool few_keys(const Range &first, const Range &last) { return min(first.hi - first.lo, last.hi - last.lo) + 1 < kFewKeys; }

// cu[s] inside [0, T], whatever the caller's array holds
__device__ __forceinline__ int token_at(const Args &a, int s) { return min(max(a.cu[s], 0), a.T); }

// The last sequence s for which begins(s, cu[s]) holds (it does for 0, and up to some s), and its tokens [first, first + count).  64
// lanes look at one sequence each: one load for up to 63 sequences, two for 4032.
struct Sequence {
  int s, first, count;
  template <typename F>
  __device__ __forceinline__ Sequence(const Args &a, int lane, F &&begins)
  {
    int at = 0, k = 64;
    for (int block = 0; a.S > 63 && block < a.S && k == 64; block += 63 * 64) {
      const int i = min(block + 63 * lane, a.S);
      const bool in = begins(i, token_at(a, i)) && i < a.S;
      k = __builtin_popcountll(__ballot(in));
      if (k > 0) at = block + 63 * (k - 1);
    }
    const int i = min(at + lane, a.S), cu = token_at(a, i);
    const bool in = begins(i, cu) && i < a.S && lane < 63;
    k = max(__builtin_popcountll(__ballot(in)), 1);  // (1 at least, if cu ascends)
    s = at + k - 1;
    first = __builtin_amdgcn_readlane(cu, k - 1);
    count = max(__builtin_amdgcn_readlane(cu, k) - first, 0);
  }
};

// inclusive sums over the lanes of a wavefront
__device__ __forceinline__ int wave_scan(int x)
{
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 to the second and fourth row, 31 to the last two
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}
// the largest of numbers >= 0
__device__ __forceinline__ int wave_max(int x)
{
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }

// The row tile that workgroup b of a key/value head takes.  A causal walk grows with the tile's place in its sequence, so the tiles of
// all sequences are taken by their place, the last places first: what sees most keys is begun first, and the workgroups of one round
// have like work (256 fp32 prompts of 20 to 200 tokens: 21.7 us in the sequences' order, 17.7 so).  C(k) = sum over sequences of
// max(tiles - k, 0) tiles stand at place k or later: the place is the largest k with C(k) > b, found by halving, 64 sequences' counts
// a register.  Under `least` sequences, whose tiles are best begun together because they read the same keys, and over kOrdered:
// in the sequences' order, from the last tile on.
constexpr int kOrdered = 256;
struct RowTile {
  int s, tok0, count, row0;  // sequence, its first token, its tokens; the tile's first row (-1: no tile)
  __device__ __forceinline__ RowTile(const Args &a, int lane, int b, int rows, int least)
  {
    if (a.S < least || a.S > kOrdered) {
      const int tile = a.row_tiles - 1 - b;
      const Sequence seq(a, lane, [&](int i, int cu) { return (int)((unsigned)(cu * a.R) / rows) + i <= tile; });
      s = seq.s;
      tok0 = seq.first;
      count = seq.count;
      row0 = (tile - (int)((unsigned)(tok0 * a.R) / rows) - s) * rows;
      if (row0 < 0 || row0 >= count * a.R) row0 = -1;
      return;
    }
    s = tok0 = count = 0;
    row0 = -1;
    if (a.S <= 64) find<1>(a, lane, b, rows);
    else find<kOrdered / 64>(a, lane, b, rows);
  }

 private:
  template <int N>
  __device__ __forceinline__ void find(const Args &a, int lane, int b, int rows)
  {
    int cu[N], n[N], t[N], most = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = 64 * i + lane;
      cu[i] = token_at(a, min(at, a.S));
      n[i] = max(token_at(a, min(at + 1, a.S)) - cu[i], 0);
      t[i] = (unsigned)(n[i] * a.R + rows - 1) / rows;
      most = max(most, t[i]);
    }
    auto beyond = [&](int k) __attribute__((always_inline)) {
      int x = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) x += max(t[i] - k, 0);
      return wave_sum(x);
    };
    if (beyond(0) <= b) return;
    int lo = 0, hi = wave_max(most);
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (beyond(mid) > b) lo = mid;
      else hi = mid;
    }
    int nth = b - beyond(lo + 1);  // of the sequences that have a tile at this place
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const unsigned long long has = __ballot(t[i] > lo);
      const int many = __builtin_popcountll(has);
      if (nth >= 0 && nth < many) {
        const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(has >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)has, 0));
        const int l = __builtin_ctzll(__ballot((has >> lane & 1ull) != 0ull && before == nth));
        s = 64 * i + l;
        tok0 = __builtin_amdgcn_readlane(cu[i], l);
        count = __builtin_amdgcn_readlane(n[i], l);
        row0 = lo * rows;
      }
      nth -= many;
    }
  }
};

}  // namespace paged
}  // namespace blossom
