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
  const int64_t *tree;         // drafted trees: [T] which of its sequence's drafted tokens a token sees, or nullptr
  int tree_rows;               // trees: rows of a workgroup: which kernel takes the call (16; shared_waves * 16; 128 or 256)
  int units;                   // workgroups a key/value head; `parts` is their number too where walks are cut (0: they are whole)
  int slots;                   // places of partial sums, [slots, G, rows of a tile, ..]
  int4 *part_at;               // [1 + T] tiles of a workgroup's share; of a token's tree, where its walks begin, tiles of one, its first row
                               // tile, its first token; in the workspace
};

// HIP counts a launch's threads in 32 bits.  The launchers below start nothing and return false for a call that would have more.
inline bool countable(long workgroups, int threads) { return workgroups * threads < 1l << 32; }

// append: paged_append.hip (a.tree: drafted tokens, turned by their places in their trees)
bool launch_append(const Args &a, hipStream_t st);
// one-token and prompt attention: paged_attn.hip.  decode_parts, prompt_parts: what `parts` is for this shape
int decode_parts(const Args &a);
int prompt_parts(const Args &a);
bool launch_decode(const Args &a, hipStream_t st);
bool launch_prompt(const Args &a, hipStream_t st);
// attention of drafted trees: paged_attn.hip.  plan_tree sets `parts` and `units`; partial results then have that many rows
void plan_tree(Args &a);
size_t tree_part_rows(const Args &a);
bool launch_tree(const Args &a, hipStream_t st);
// accepted drafts, forked sequences, copied pages: paged_pages.hip
struct Accept {
  const int *keep;             // [S, width] ascending drafted tokens, up to the first entry that is none
  int width;
  int *new_len;                // [S] or nullptr
};
bool launch_accept(const Args &a, const Accept &x, hipStream_t st);
struct Fork {
  int N, grow;                 // new sequences; positions that each gets room for
  const int *parent;           // [N]
  const int *refs;             // [n_pages] who holds a page
  int *table, *len, *new_refs; // [N, max_pages], [N], [n_pages]
  int *copies, *missing;       // [N, 3] source, target, rows; [1]
  int4 *at;                    // [N] a sequence's first fresh page, its last one where it keeps pages among them (else below 0), page and rows
                               // that it copies (below 0: none; to its first fresh page); in the workspace
  uint4 *asks;                 // [N, chunks] of the row of one that does, 64 entries at a time, which are fresh (low, high bits), and how many before
                               // these are, there too
  int chunks;
  int *fresh;                  // [N] pages that it gets, there too
  int *held;                   // [n_pages] does a copy read a page, there too
};
bool launch_fork(const Args &a, const Fork &x, hipStream_t st);
bool launch_copy(const Args &a, const int *copies, int count, hipStream_t st);
// prompt attention for bf16, d = 64 or 128: paged_prompt.hip
constexpr int kPromptRows = 128;  // query rows of a workgroup, which has four wavefronts
constexpr int kPromptWaves = 4;
bool prompt_mfma_supported(const Args &a);
void launch_prompt_mfma(const Args &a, hipStream_t st);
// prompt attention for everything else: paged_shared.hip
// rows of a workgroup: 16 a wavefront, of which there are as many as it takes to move a tile
constexpr int shared_waves(int row_bytes) { return row_bytes >= 256 ? 4 : 2; }
void launch_prompt_shared(const Args &a, hipStream_t st);
// the same for drafted trees
void launch_tree_shared(const Args &a, hipStream_t st);
// drafted trees of more than 16 rows for bf16, d = 64 or 128: paged_tree.hip (once: loads past the caches)
bool tree_matrix_supported(const Args &a);
void launch_tree_matrix(const Args &a, bool once, hipStream_t st);

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

// ---- drafted trees ----
//
// The n drafted tokens of a sequence take the slots past .. past + n - 1 after its history, token i slot past + i; bit k of its mask says
// that it sees drafted token k (k < 64, k < n).  It stands `depth` positions behind the history, the number of other drafted tokens it sees.
constexpr int kDrafts = 64;
constexpr int kTreeLeast = 512;  // keys of a workgroup's share, at least, where rows share them
__device__ __forceinline__ unsigned long long below(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }
__device__ __forceinline__ int depth_of(unsigned long long mask, int i, int n)
{
  mask &= below(n);
  if (i < 64) mask &= ~(1ull << i);
  return __builtin_popcountll(mask);
}

// What the tokens of one sequence's tree see.
struct Tree {
  int past;          // positions before the drafted tokens (below 0 if there are fewer positions than tokens: slots below 0 do not exist)
  int shown;         // drafted tokens that can be seen
  Range any, every;  // keys that any token can see; of the history those that all do
  __device__ __forceinline__ Tree(const Args &a, int raw_len, int n)
  {
    past = max(raw_len, 0) - n;
    shown = min(min(n, kDrafts), past > a.cap - kDrafts ? a.cap - past : kDrafts);
    any = {first(a, 0), past + shown - 1};
    every = {first(a, min(n - 1, kDrafts)), min(past, a.cap) - 1};  // (a token behind the 64th may see all of these)
  }
  // the first key that a token sees at this depth
  __device__ __forceinline__ int first(const Args &a, int depth) const
  {
    if (a.window == 0x7FFFFFFF) return 0;
    return (int)min(max((long)max(past, 0) + depth - a.window + 1, 0l), 0x7FFFFFFFl);
  }
};

// One token's keys, 32 at a time.
struct Seen {
  int lo;                   // of the history
  unsigned long long mask;  // of the drafted tokens
  Seen() = default;
  __device__ __forceinline__ Seen(const Args &a, const Tree &t, unsigned long long given, int i, int n)
  {
    lo = t.first(a, depth_of(given, i, n));
    mask = given & below(t.shown);
  }
  template <typename F>
  __device__ __forceinline__ unsigned bits(const Tree &t, int base, F &&row_bits) const
  {
    const int to = base - t.past;  // the drafted token at key `base`
    const unsigned drafted = to >= 64 || to <= -32 ? 0u : to >= 0 ? (unsigned)(mask >> to) : (unsigned)(mask << -to);
    return row_bits(lo - base, t.every.hi - base) | drafted;
  }
};

// Rows of one sequence and key/value head, and what is walked for them.
struct Walk {
  int s = -1, tok0 = 0, count = 0, row0 = 0;  // sequence (below 0: none), its first token, its tokens, the first row
  int len = 0;                                // trees: its kv_len
  int part = 0;                               // prompts: which part of the walk
  int from = 0, tiles = 0x7FFFFFFF;           // trees: tiles of the walk from its first on
  int slot = -1;                              // trees: where partial sums go (below 0: the walk is whole)
};

// Which workgroup of all trees' this one is.  Where a walk is one workgroup's, up to one place a sequence has nothing (launch_tree counts row
// tiles before it knows them), and with fewer than 8 key/value heads these would lie on the same dies, to which workgroups go in turn: eights
// are turned by their number (64 trees of 16 rows, 4 heads: every other row tile is nothing; 16.2 us, so 12.1).
__device__ __forceinline__ int tree_block(const Args &a)
{
  const unsigned id = blockIdx.x, eight = id & ~7u;
  return a.G >= 8 || eight + 8 > gridDim.x ? id : eight | ((id + (id >> 3)) & 7u);
}

// What one workgroup of a key/value head does of all trees.  A tree's rows are cut into row tiles, each of which walks the same key tiles.  With
// a.parts workgroups, the walks of all row tiles lie one behind the other, and workgroup b takes the b-th of as many equal shares: the end
// of one walk, whole ones, the beginning of another.  (Cut into parts by themselves, 16 walks of 125 to 253 tiles leave the longest part
// 1.5 to 1.8 times the mean.)  Row tile j's part in workgroup b has slot b + j.  Otherwise (a.parts 0) a workgroup takes one walk.
struct TreeWork {
  struct One {
    int cu, n, len, tiles, row_tiles;
  };
  int unit, rows, keys;  // workgroup; rows of a row tile, keys of a tile
  int at = 0, end = 0, share = 0;
  __device__ __forceinline__ One look(const Args &a, int i) const
  {
    One x{token_at(a, min(i, a.S)), 0, 0, 0, 0};
    if (i >= a.S) return x;
    x.len = a.kv_len[i];
    x.n = max(token_at(a, i + 1) - x.cu, 0);
    if (x.n == 0) return x;
    const Tree t(a, x.len, x.n);
    x.tiles = t.any.hi >= t.any.lo ? t.any.hi / keys - t.any.lo / keys + 1 : 1;  // (a walk of nothing has a place too)
    x.row_tiles = (unsigned)(x.n * a.R + rows - 1) / rows;
    return x;
  }
  __device__ __forceinline__ TreeWork(int unit, int rows, int keys) : unit(unit), rows(rows), keys(keys) {}
  // The first walk.
  __device__ __forceinline__ Walk begin(const Args &a, int lane, int least)
  {
    if (a.parts == 0) {
      Walk w;
      const Sequence seq(a, lane, [&](int i, int cu) { return (int)((unsigned)(cu * a.R) / rows) + i <= unit; });
      const int row0 = (unit - (int)((unsigned)(seq.first * a.R) / rows) - seq.s) * rows;
      if (row0 < 0 || row0 >= seq.count * a.R) return w;
      w.s = seq.s; w.tok0 = seq.first; w.count = seq.count; w.row0 = row0;
      w.len = __builtin_amdgcn_readfirstlane(a.kv_len[w.s]);
      return w;
    }
    const One mine0 = look(a, lane);
    int total = 0, walks = 0;
    for (int s0 = 0; s0 < a.S; s0 += 64) {
      const One x = s0 == 0 ? mine0 : look(a, s0 + lane);
      total += wave_sum(x.tiles * x.row_tiles);
      walks += wave_sum(x.row_tiles);
    }
    // `least` tiles, or a walk of the mean length: shorter ones are not gathered in few workgroups where the caller grants far more than is used
    // (100 trees of 16 rows over 100 positions, tables for 131072: 32 us, so 12.3; tables for 112: 8.1)
    const unsigned mean = (unsigned)(total + walks - 1) / (unsigned)max(walks, 1);
    share = max(max((unsigned)(total + a.parts - 1) / (unsigned)a.parts, min((unsigned)least, mean)), 1u);
    at = (int)min((long)unit * share, (long)total);
    end = (int)min((long)at + share, (long)total);
    return take(a, lane, mine0);
  }
  // The next walk, or piece of one (s < 0: no more).  The first workgroup of a key/value head tells the join where each tree lies.
  __device__ __forceinline__ Walk next(const Args &a, int lane)
  {
    if (at >= end) return Walk{};
    return take(a, lane, look(a, lane));
  }
  __device__ __forceinline__ Walk take(const Args &a, int lane, const One &mine0)
  {
    Walk w;
    if (at >= end) return w;
    int done = 0, tiles_done = 0;  // row tiles, and tiles of their walks
    for (int s0 = 0; s0 < a.S; s0 += 64) {
      const One x = s0 == 0 ? mine0 : look(a, s0 + lane);
      const int mine = x.tiles * x.row_tiles, upto = tiles_done + wave_scan(mine), row_upto = done + wave_scan(x.row_tiles);
      const int k = __builtin_popcountll(__ballot(upto <= at));
      if (k < 64) {
        const int tiles = __builtin_amdgcn_readlane(x.tiles, k), row_tiles = __builtin_amdgcn_readlane(x.row_tiles, k);
        const int in = at - (__builtin_amdgcn_readlane(upto, k) - tiles * row_tiles), tile = (unsigned)in / (unsigned)tiles;
        const int to = unit + __builtin_amdgcn_readlane(row_upto, k) - row_tiles + tile;
        if ((unsigned)tile >= (unsigned)row_tiles || (unsigned)to >= (unsigned)a.slots) {  // (cu_seqlens does not ascend)
          at = end;
          return w;
        }
        w.s = s0 + k;
        w.tok0 = __builtin_amdgcn_readlane(x.cu, k);
        w.count = __builtin_amdgcn_readlane(x.n, k);
        w.len = __builtin_amdgcn_readlane(x.len, k);
        w.row0 = tile * rows;
        w.from = in - tile * tiles;
        w.tiles = min(end - at, tiles - w.from);
        if (w.tiles < tiles) w.slot = to;
        at += w.tiles;
        return w;
      }
      tiles_done = __builtin_amdgcn_readlane(upto, 63);
      done = __builtin_amdgcn_readlane(row_upto, 63);
    }
    return w;
  }
  // By the workgroup that has a tree's first piece: for the join.
  __device__ __forceinline__ void tell(const Args &a, const Walk &w, int g, int lane, int tid, int threads) const
  {
    if (a.parts == 0 || w.row0 != 0 || w.from != 0 || g != 0) return;
    int done = 0, tiles_done = 0;
    for (int s0 = 0; s0 < a.S; s0 += 64) {
      const One x = look(a, s0 + lane);
      const int upto = tiles_done + wave_scan(x.tiles * x.row_tiles), row_upto = done + wave_scan(x.row_tiles);
      if (w.s < s0 + 64) {
        const int k = w.s - s0, tiles = __builtin_amdgcn_readlane(x.tiles, k), row_tiles = __builtin_amdgcn_readlane(x.row_tiles, k);
        const int4 place = make_int4(__builtin_amdgcn_readlane(upto, k) - tiles * row_tiles, tiles, __builtin_amdgcn_readlane(row_upto, k) - row_tiles, w.tok0);
        for (int i = tid; i < w.count; i += threads) a.part_at[1 + w.tok0 + i] = place;
        if (tid == 0) a.part_at[0] = make_int4(share, 0, 0, 0);  // (all that write it write the same)
        return;
      }
      tiles_done = __builtin_amdgcn_readlane(upto, 63);
      done = __builtin_amdgcn_readlane(row_upto, 63);
    }
  }
};

}  // namespace paged
}  // namespace blossom
