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

// append: paged_append.hip
void launch_append(const Args &a, hipStream_t st);
// one-token and prompt attention: paged_attn.hip.  decode_parts, prompt_parts: what `parts` is for this shape
int decode_parts(const Args &a);
int prompt_parts(const Args &a);
void launch_decode(const Args &a, hipStream_t st);
void launch_prompt(const Args &a, hipStream_t st);
// prompt attention for bf16, d = 64 or 128: paged_prompt.hip
constexpr int kPromptRows = 128;  // query rows of a workgroup
bool prompt_mfma_supported(const Args &a);
void launch_prompt_mfma(const Args &a, hipStream_t st);
// prompt attention for everything else: paged_shared.hip
constexpr int kSharedRows = 64;
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

// Keys lo .. hi that a query at `pos` sees, of a sequence with n keys (hi < lo: none).
struct Range {
  int lo, hi;
};
__device__ __forceinline__ Range seen_by(const Args &a, int pos, int n)
{
  if (pos < 0) return {0, -1};
  return {max(pos - a.window + 1, 0), min(pos, min(n, a.cap) - 1)};
}

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

}  // namespace paged
}  // namespace blossom
