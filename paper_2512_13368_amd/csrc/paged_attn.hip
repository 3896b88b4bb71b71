// Attention over a paged key/value cache: one new token a sequence (decode), or a run of new tokens (prompt).
//
//   o = sum_j p_j V_j,  p = softmax_j(scale q.K_j)   over the cached positions j that the query sees:
//   j <= pos, pos - j < window, pos = kv_len - new + i for new token i (decode: pos = kv_len - 1)
//
// Query rows are (token, head) pairs that share a key/value head: the R = H/G heads of a token read the same keys, so they stand in
// one 16-row operand.  This file has the way through a cache that memory bounds, one new token a sequence or a few: the wavefronts
// of a workgroup take a run of its 32-key tiles each, through LDS that is theirs alone (no barrier in the walk), and join their
// results there.  Where a sequence is long and workgroups are few, its keys are cut into parts for several, whose results a second
// kernel joins.  Large prompts: paged_prompt.hip, paged_shared.hip.  The operands and the softmax of a step: paged_tile.h.
//
// Measured: one sequence of 131071 keys (32 heads over 8, d = 128, bf16: 537 MB) 86 us, 80 of it in this kernel, where reading as many
// bytes takes 78; 16 sequences of 4001 to 8191 keys (400 MB) 72 us, the join 4.6 of it; 128 of 100 to 1024 (4 heads, d = 64: 74 MB)
// 15.4 us, where a read takes 11 and a launch with its first loads 4; the join inside the kernel would save 3 us of 85 and nothing
// where sequences are short.
#include "common.h"
#include "launch.h"
#include "mfma_common.h"
#include "paged.h"
#include "paged_tile.h"

namespace blossom {
namespace paged {

namespace {

using mfma::kLn2;
using mfma::kNegInf;

constexpr int kRows = 16;             // query rows of a workgroup
constexpr int kMostParts = 256;       // parts of a key/value head's keys, of all sequences together
constexpr int kMostPromptParts = 64;  // parts of a row's keys in a prompt
// Decode wavefronts that keep the memory busy: two a SIMD (four: 88 us for 85 at 131071 keys, 16.0 for 15.2 on short ones).  Four where rows
// are small, which take as long to work on (67201 keys with a window of 29264, 3 sequences, 8 heads, fp32, d = 8: 20 us for 28.5; 13 of
// 1462 to 14625, 32 heads over 4, bf16, d = 32: 17.1 for 18.4), one where a CU's LDS holds no more (131000 keys, 8 heads over 2, fp32,
// d = 128: 59 for 65; 20106 for 2 sequences, 6 over 2: 24 for 35).
constexpr int fill_waves(int row_bytes) { return row_bytes <= 64 ? 4096 : row_bytes <= 256 ? 2048 : 1024; }
// A wavefront's tiles from which splitting a sequence pays for the join (8 heads over 2, d = 128, one sequence: 32 tiles over 8
// wavefronts 8.8 us whole and 10.8 split, 63 tiles 13.9 and 10.8; fp32 at d = 32: 9.4 and 11.0, 16.9 and 12.1).  Large fp32 rows, whose tiles
// take longest, from 4 on (4 sequences, 8 heads over 4: 500 keys at d = 128 16.8 and 14.4, 1000 at d = 64 14.5 and 13.4).
constexpr int split_tiles(int dtype, int d) { return dtype == 0 && d >= 64 ? 4 : 6; }

enum PromptKind { kFew, kShared, kMatrix };
struct PromptPlan {
  PromptKind kind;
  int parts;
};

}  // namespace

// A wavefront of decode holds two tiles of K and of V in LDS, one on its way; of tiles of 16 KB and more one alone, eight wavefronts
// (or four) to a CU.  (At d = 128, bf16: four wavefronts of two tiles 86.5 us for 131071 keys, eight of one 85.6; two of four
// 111.)  A workgroup's wavefronts take up to 128 KB.
constexpr int decode_stages(int row_bytes) { return row_bytes >= 256 ? 1 : 2; }
constexpr int most_decode_waves(int row_bytes)
{
  const int held = decode_stages(row_bytes) * 2 * (row_bytes < 32 ? 1024 : 32 * row_bytes);
  return 131072 / held < 16 ? 131072 / held : 16;
}

// Four wavefronts at least; one round of workgroups of the most is no more than kMostParts.
constexpr bool fits_parts(int row_bytes)
{
  return most_decode_waves(row_bytes) >= 4 && fill_waves(row_bytes) / most_decode_waves(row_bytes) <= kMostParts;
}
static_assert(fits_parts(16) && fits_parts(32) && fits_parts(64) && fits_parts(128) && fits_parts(256) && fits_parts(512), "");

// ---- work of decode, split over a long cache ----
__device__ __forceinline__ int tiles_of(const Args &a, int s)
{
  if (s >= a.S) return 0;
  const int len = max(a.kv_len[s], 0);
  const Range r = seen_by(a, len - 1, len);
  return r.hi >= r.lo ? r.hi / kTile - r.lo / kTile + 1 : 0;
}
// The part of all sequences' keys that workgroup b of a key/value head takes: of a.parts workgroups, a sequence of t tiles is cut into
// ceil(t / chunk), so that ragged lengths give parts of like size.  Every wavefront finds its own from the lengths, 64 sequences at a
// time: a chunk of total / (parts - S / 2) nearly always makes few enough parts (half a part a sequence is lost to rounding up), one
// of total / (parts - S) always does.
struct Part {
  int s = -1, first = 0, count = 0;  // sequence (-1: none), its first part, its parts
  __device__ __forceinline__ Part(const Args &a, int lane, int b, int least)
  {
    const int t0 = tiles_of(a, lane);
    auto tiles = [&](int s0) { return s0 == 0 ? t0 : tiles_of(a, s0 + lane); };
    int total = 0;
    for (int s0 = 0; s0 < a.S; s0 += 64) total += wave_sum(tiles(s0));
    int chunk = max((total + a.parts - a.S / 2 - 1) / (a.parts - a.S / 2), least);
    auto cut = [&](int t) { return (int)(((float)t + (float)(chunk - 1) + 0.5f) / (float)chunk); };  // ceil(t / chunk)
    int need = 0;
    for (int s0 = 0; s0 < a.S; s0 += 64) need += wave_sum(cut(tiles(s0)));
    if (need > a.parts) chunk = max((total + a.parts - a.S - 1) / (a.parts - a.S), least);
    int done = 0;
    for (int s0 = 0; s0 < a.S; s0 += 64) {
      const int mine = cut(tiles(s0)), upto = done + wave_scan(mine);
      const int k = __builtin_popcountll(__ballot(upto <= b));
      if (k < 64) {
        s = s0 + k;
        count = __builtin_amdgcn_readlane(mine, k);
        first = __builtin_amdgcn_readlane(upto, k) - count;
        return;
      }
      done = __builtin_amdgcn_readlane(upto, 63);
    }
  }
};

// What a workgroup of the kernels below takes: up to 16 rows that share keys, and which part of their walk.
struct FewRows {
  int s, row0, rows, tok0, new_tokens = 1, part = 0, n_parts = 1, b = 0;
};

// One new token a sequence, or few (PROMPT; TREE: drafted ones): W wavefronts take a run of key tiles each for up to 16 rows that share
// keys.  SPLIT: of a part of them.
template <typename T, int D, int W, bool ONCE, bool SPLIT, bool PROMPT, bool TREE>
__device__ __forceinline__ void few_rows(const Args &a, int g, const FewRows &mine_rows, const Walk &walk)
{
  typedef Tile<T, D> TL;
  constexpr int STAGES = decode_stages(TL::RB), HOLD = STAGES * 2 * TL::BYTES;  // LDS of a wavefront
  constexpr int LDR = D + 4;  // floats of a row of results
  static_assert(kRows * LDR * 4 <= HOLD, "results go where the tiles were");
  __shared__ __attribute__((aligned(1024))) char lds[W * HOLD];
  __shared__ float m_s[W][kRows], l_s[W][kRows];
  int lane = threadIdx.x & 63;
  if constexpr (TREE) asm volatile("" : "+v"(lane));  // (what depends on it is not kept in registers from one walk to the next)
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, c = lane >> 4;
  const int s = mine_rows.s, row0 = mine_rows.row0, rows = mine_rows.rows, tok0 = mine_rows.tok0, new_tokens = mine_rows.new_tokens;
  const int part = mine_rows.part, n_parts = mine_rows.n_parts, b = mine_rows.b;
  const int row = row0 + min(n, rows - 1), tok = PROMPT ? a.by_R.of(row) : 0, head = g * a.R + row - tok * a.R;

  // what hangs on nothing is requested before anything is waited for: the length, the query, the first pages
  const int *table = a.page_table + s * a.table_seq + g * a.table_group;
  auto entries = [&](int first) __attribute__((always_inline)) -> int {
    const int id = table[min(first + lane, a.max_pages - 1)];
    return id >= 0 && id < a.n_pages ? id : -1;
  };
  const int raw_len = TREE ? walk.len : a.kv_len[s];
  int list0 = 0, ids = entries(0);  // pages list0 .. list0 + 63, one a lane
  typename TL::Query q;
  TL::load_query(q, static_cast<const T *>(a.Q) + (tok0 + tok) * a.q_stride + (size_t)head * D, c);
  unsigned long long mask = 0ull;
  if constexpr (TREE) mask = a.tree[tok0 + tok];

  const int len = max(__builtin_amdgcn_readfirstlane(raw_len), 0);
  const int first_pos = len - new_tokens;
  const Tree tree(a, len, new_tokens);
  const Seen sees(a, tree, mask, tok, new_tokens);
  // keys that any row sees, that this lane's row does, that all do
  Range any = TREE ? tree.any : seen_by(a, first_pos + (PROMPT ? a.by_R.of(row0) : 0), len), my = any, every = TREE ? tree.every : any;
  if constexpr (PROMPT && !TREE) {
    const Range last = seen_by(a, first_pos + a.by_R.of(row0 + rows - 1), len);
    every.lo = last.lo;
    any.hi = last.hi;
    my = seen_by(a, first_pos + tok, len);
  }
  const int t_lo = any.lo / kTile, t_all = any.hi >= any.lo ? any.hi / kTile - t_lo + 1 : 0;
  int t_begin = t_lo, t_end = t_lo + t_all;
  if constexpr (TREE) {
    t_begin = t_lo + min(walk.from, t_all);
    t_end = t_begin + min(walk.tiles, t_lo + t_all - t_begin);
  } else if constexpr (SPLIT) {
    const int each = (t_all + n_parts - 1) / n_parts;
    t_begin = t_lo + min(part * each, t_all);
    t_end = t_lo + min((part + 1) * each, t_all);
  }
  const int run = (t_end - t_begin + W - 1) / W;
  int t = min(t_begin + wv * run, t_end);
  const int t_stop = min(t + run, t_end);

  char *mine = lds + wv * HOLD;
  const size_t page_bytes = ((size_t)a.G << a.page_shift) * TL::RB, group_bytes = ((size_t)g << a.page_shift) * TL::RB;
  auto request = [&](int t, char *to) __attribute__((always_inline)) -> unsigned {
    const int first = (t * kTile) >> a.page_shift, last = (t * kTile + kTile - 1) >> a.page_shift;
    if (first < list0 || last >= list0 + 64) {
      list0 = first;
      ids = entries(first);
    }
    const int key = t * kTile + (lane & 31);
    const int id = __shfl(ids, (key >> a.page_shift) - list0);
    const bool ok = id >= 0 && key >= any.lo && key <= any.hi;
    const unsigned seen = (unsigned)__ballot(ok);
    const size_t off = max(id, 0) * page_bytes + group_bytes + (size_t)(key & ((1 << a.page_shift) - 1)) * TL::RB;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (what was read from `to` is here)
    TL::template request<ONCE>(a, to, to + TL::BYTES, off, ok, seen == 0xFFFFFFFFu, lane, 0, 1);
    return seen;
  };

  Rows<T, D> r;
  r.clear();
  // a ring of STAGES tiles: those of the next STAGES - 1 are on their way while one is worked on
  unsigned seen[STAGES];
#pragma unroll
  for (int k = 0; k < STAGES - 1; ++k) seen[k] = t + k < t_stop ? request(t + k, mine + k * (2 * TL::BYTES)) : 0u;
  while (t < t_stop) {
#pragma unroll
    for (int k = 0; k < STAGES; ++k) {
      if (t >= t_stop) break;
      constexpr int AHEAD = STAGES - 1;
      const int to = (k + AHEAD) % STAGES;
      if (t + AHEAD < t_stop) {
        seen[to] = request(t + AHEAD, mine + to * (2 * TL::BYTES));
        arrived<2 * TL::LOADS * AHEAD>();
      } else {
        arrived<0>();
      }
      const char *ks = mine + k * (2 * TL::BYTES);
      const int base = t * kTile;
      const bool all = seen[k] == 0xFFFFFFFFu && (!PROMPT || (base >= every.lo && base + kTile - 1 <= every.hi));
      const unsigned row = TREE ? sees.bits(tree, base, mfma::row_bits) : PROMPT ? mfma::row_bits(my.lo - base, my.hi - base) : 0xFFFFFFFFu;
      r.template attend<true>(ks, ks + TL::BYTES, q, a.scale2, seen[k] & row, all, true, lane);
      ++t;
    }
  }

  // ---- the wavefronts' results ----
  const float l = r.total();
  if (n < rows) {
    if (c == 0) {
      m_s[wv][n] = r.m;
      l_s[wv][n] = l;
    }
    float *to = reinterpret_cast<float *>(mine) + n * LDR;
#pragma unroll
    for (int j = 0; j < TL::NV; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (TL::channel(j, c, i) < D) to[TL::channel(j, c, i)] = r.acc[j][i];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < rows * (D / 4); e += 64 * W) {
    const int row = e / (D / 4), ch = e % (D / 4) * 4;
    float mm = kNegInf;
#pragma unroll
    for (int w = 0; w < W; ++w) mm = fmaxf(mm, m_s[w][row]);
    const float ref = mm == kNegInf ? 0.0f : mm;
    float ll = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = __builtin_amdgcn_exp2f(m_s[w][row] - ref);
      const float4 v = *reinterpret_cast<const float4 *>(lds + w * HOLD + (row * LDR + ch) * 4);
      ll = fmaf(l_s[w][row], f, ll);
      o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
    }
    const int tk = PROMPT ? a.by_R.of(row0 + row) : 0;
    const size_t out = (size_t)(tok0 + tk) * a.H + g * a.R + row0 + row - tk * a.R;
    if (!SPLIT || (TREE ? walk.slot < 0 : !PROMPT && n_parts == 1)) {
      const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
      store_four(static_cast<T *>(a.O) + out * D + ch, o, inv);
      if (ch == 0 && a.lse) a.lse[out] = ll == 0.0f ? kNegInf : (mm + __log2f(ll)) * kLn2;
    } else {  // decode: [heads of the token][parts of all sequences]; prompt: [rows][parts of each]; trees: [slots][heads][rows of a tile]
      const size_t at = TREE ? ((size_t)walk.slot * a.G + g) * kRows + row : PROMPT ? out * a.parts + part : (size_t)(g * a.R + row0 + row) * a.parts + b;
      *reinterpret_cast<float4 *>(a.part_o + at * D + ch) = o;
      if (ch == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(mm, ll);
    }
  }
}

template <typename T, int D, int W, bool ONCE, bool SPLIT, bool PROMPT>
__global__ __launch_bounds__(64 * W) void decode_kernel(Args a)
{
  const int lane = threadIdx.x & 63, rest = a.by_G.of(blockIdx.x), g = blockIdx.x - rest * a.G;
  FewRows r;
  if constexpr (PROMPT) {
    const int tile = a.by_parts.of(rest);
    r.part = rest - tile * a.parts;
    r.n_parts = a.parts;
    const Sequence seq(a, lane, [&](int i, int cu) { return (int)((unsigned)(cu * a.R) / kRows) + i <= tile; });
    r.s = seq.s;
    r.tok0 = seq.first;
    r.new_tokens = seq.count;
    r.row0 = (tile - (int)((unsigned)(r.tok0 * a.R) / kRows) - r.s) * kRows;
    if (r.row0 < 0 || r.row0 >= r.new_tokens * a.R) return;
    r.rows = min(r.new_tokens * a.R - r.row0, kRows);
  } else {
    const int tiles = (a.R + kRows - 1) / kRows;
    r.b = tiles == 1 ? rest : rest / tiles;
    r.row0 = (rest - r.b * tiles) * kRows;
    r.s = r.b;
    if constexpr (SPLIT) {
      const Part mine(a, lane, r.b, W);
      if (mine.s < 0) return;
      r.s = mine.s;
      r.part = r.b - mine.first;
      r.n_parts = mine.count;
      if (r.part == 0 && g == 0 && r.row0 == 0 && threadIdx.x == 0) a.part_of[r.s] = make_int2(mine.first, r.n_parts);  // for the join
    }
    r.tok0 = r.s;
    r.rows = min(a.R - r.row0, kRows);
  }
  few_rows<T, D, W, ONCE, SPLIT, PROMPT, false>(a, g, r, Walk{});
}

template <typename T, int D, int W, bool SPLIT>
__global__ __launch_bounds__(64 * W) void tree_few_kernel(Args a)
{
  const int lane = threadIdx.x & 63, block = tree_block(a), rest = a.by_G.of(block), g = block - rest * a.G;
  TreeWork work(rest, kRows, kTile);
  for (Walk w = work.begin(a, lane, W); w.s >= 0; w = work.next(a, lane)) {
    work.tell(a, w, g, lane, threadIdx.x, 64 * W);
    FewRows r;
    r.s = w.s; r.tok0 = w.tok0; r.new_tokens = w.count; r.row0 = w.row0;
    r.rows = min(w.count * a.R - w.row0, kRows);
    few_rows<T, D, W, false, SPLIT, true, true>(a, g, r, w);
    __syncthreads();
  }
}

// Joins the parts of a sequence's row, where it has more than one: a workgroup a row, whose threads take a part each for the weights
// and then, 4 channels each, every (256 / (d / 4))-th part's sums.  Parts that met no key have weight 0 and finite sums.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_kernel(Args a)
{
  constexpr int LANES = D / 4, GROUPS = 256 / LANES;
  __shared__ float red_s[4], l_s[4], w_s[kMostParts];
  __shared__ __attribute__((aligned(16))) float o_s[GROUPS][D];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  T *O = static_cast<T *>(a.O) + (size_t)blockIdx.x * D;
  const int s = a.by_H.of(blockIdx.x), h = blockIdx.x - s * a.H;
  const int2 part = a.part_of[s];  // (of a sequence without keys: whatever the workspace held)
  const int n = __builtin_amdgcn_readfirstlane(tiles_of(a, s) > 0 ? part.y : 0);
  if (n <= 1) {
    if (n == 1) return;  // (the part's workgroup wrote the row)
    if (tid < D) store_out(O + tid, 0.0f);
    if (tid == 0 && a.lse) a.lse[blockIdx.x] = kNegInf;
    return;
  }
  const size_t at0 = (size_t)h * a.parts + part.x;
  const float *ml = a.part_ml + at0 * 2;
  const float4 *po = reinterpret_cast<const float4 *>(a.part_o + at0 * D);
  const int at = tid % LANES, grp = tid / LANES;
  float4 early[8];  // (requested with the weights)
#pragma unroll
  for (int k = 0; k < 8; ++k)
    early[k] = grp + k * GROUPS < n ? po[(size_t)(grp + k * GROUPS) * LANES + at] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const bool mine = tid < n;
  const float2 x = mine ? *reinterpret_cast<const float2 *>(ml + 2 * tid) : make_float2(kNegInf, 0.0f);
  float m = x.x;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if (lane == 0) red_s[wv] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red_s[0], red_s[1]), fmaxf(red_s[2], red_s[3]));
  const float w = __builtin_amdgcn_exp2f(x.x - (m == kNegInf ? 0.0f : m));
  float l = x.y * w;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) l += __shfl_xor(l, o);
  w_s[tid] = mine ? w : 0.0f;
  if (lane == 0) l_s[wv] = l;
  __syncthreads();
  l = (l_s[0] + l_s[1]) + (l_s[2] + l_s[3]);
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  auto add = [&](const float4 &v, float f) __attribute__((always_inline)) {
    o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
  };
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (grp + k * GROUPS < kMostParts) add(early[k], w_s[grp + k * GROUPS]);
  for (int i = grp + 8 * GROUPS; i < n; i += GROUPS) add(po[(size_t)i * LANES + at], w_s[i]);
  *reinterpret_cast<float4 *>(&o_s[grp][4 * at]) = o;
  __syncthreads();
  if (tid < D) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) sum += o_s[i][tid];
    store_out(O + tid, l == 0.0f ? 0.0f : sum / l);
  }
  if (tid == 0 && a.lse) a.lse[blockIdx.x] = l == 0.0f ? kNegInf : (m + __log2f(l)) * kLn2;
}

// Joins the parts of prompt rows: D / 4 threads a row, 4 channels each, every part's weight computed by all of them.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_rows_kernel(Args a)
{
  constexpr int LANES = D / 4, ROWS = 256 / LANES, AHEAD = 8;
  const int at = threadIdx.x % LANES;
  const size_t row = (size_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (row >= (size_t)token_at(a, a.S) * a.H) return;  // (a row that no sequence owns stays as it is)
  const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + row * a.parts;
  const float4 *po = reinterpret_cast<const float4 *>(a.part_o) + row * a.parts * LANES + at;
  float m = kNegInf;
  for (int i = 0; i < a.parts; ++i) m = fmaxf(m, ml[i].x);
  const float ref = m == kNegInf ? 0.0f : m;
  float l = 0.0f;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int i = 0; i < a.parts; i += AHEAD) {
    float4 v[AHEAD];
    float2 x[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int j = min(i + k, a.parts - 1);
      v[k] = po[(size_t)j * LANES];
      x[k] = ml[j];
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const float w = i + k < a.parts ? __builtin_amdgcn_exp2f(x[k].x - ref) : 0.0f;
      l = fmaf(x[k].y, w, l);
      o.x = fmaf(v[k].x, w, o.x); o.y = fmaf(v[k].y, w, o.y); o.z = fmaf(v[k].z, w, o.z); o.w = fmaf(v[k].w, w, o.w);
    }
  }
  store_four(static_cast<T *>(a.O) + row * D + 4 * at, o, l == 0.0f ? 0.0f : 1.0f / l);
  if (at == 0 && a.lse) a.lse[row] = l == 0.0f ? kNegInf : (m + __log2f(l)) * kLn2;
}

// Joins the parts of drafted tokens' rows, where a walk has more than one.  D / 4 lanes have 4 channels each of a part; GROUPS such groups
// take a row's parts in turn, and are summed over at the end.  `rows`: of a workgroup of the walk.  One group has two or three parts as a
// rule, and requests three at once (24832 rows of d = 128, 36 MB: 10.3 us, eight at once 12.9).
template <typename T, int D, int GROUPS>
__global__ __launch_bounds__(256) void join_tree_kernel(Args a, int rows)
{
  constexpr int LANES = D / 4, EACH = LANES * GROUPS, ROWS = 256 / EACH, AHEAD = GROUPS > 1 ? 8 : 3;
  __shared__ float4 o_s[GROUPS > 1 ? 256 : 1];
  __shared__ float2 ml_s[GROUPS > 1 ? 256 / LANES : 1];
  const int at = threadIdx.x % LANES, grp = threadIdx.x / LANES % GROUPS;
  const size_t row = (size_t)blockIdx.x * ROWS + threadIdx.x / EACH;
  // (a row that no sequence owns stays as it is, and one that its walk's workgroup wrote)
  int parts = 0;
  size_t step = 0, at0 = 0;
  if (row < (size_t)token_at(a, a.S) * a.H) {
    const int t = a.by_H.of((int)row), h = (int)row - t * a.H;
    const int share = a.part_at[0].x;
    const int4 of = a.part_at[1 + t];
    const int g = a.by_R.of(h), r = (t - of.w) * a.R + h - g * a.R, tile = (unsigned)r / (unsigned)rows;
    const long begin = of.x + (long)tile * of.y;  // of the row's walk, among all
    if (share > 0 && r >= 0 && begin >= 0 && of.y > 0 && begin + of.y <= 1l << 31) {  // (else cu_seqlens does not ascend: whatever the workspace held)
      const int first = (int)((unsigned)begin / (unsigned)share), last = (int)((unsigned)(begin + of.y - 1) / (unsigned)share);
      const long slot = (long)first + of.z + tile;
      if (last > first && slot >= 0 && slot + last - first < a.slots) {
        parts = last - first + 1;
        step = (size_t)a.G * rows;
        at0 = (slot * a.G + g) * rows + (r - tile * rows);
      }
    }
  }
  if (GROUPS == 1 && parts == 0) return;
  const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + at0;
  const float4 *po = reinterpret_cast<const float4 *>(a.part_o) + at0 * LANES + at;
  float m = kNegInf;
  for (int i = grp; i < parts; i += GROUPS) m = fmaxf(m, ml[i * step].x);
  const float ref = m == kNegInf ? 0.0f : m;
  float l = 0.0f;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  auto add = [&](const float4 &v, float w) __attribute__((always_inline)) {
    o.x = fmaf(v.x, w, o.x); o.y = fmaf(v.y, w, o.y); o.z = fmaf(v.z, w, o.z); o.w = fmaf(v.w, w, o.w);
  };
  for (int i = grp; i < parts; i += AHEAD * GROUPS) {
    float4 v[AHEAD];
    float2 x[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const size_t j = min(i + k * GROUPS, parts - 1) * step;
      v[k] = po[j * LANES];
      x[k] = ml[j];
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const float w = i + k * GROUPS < parts ? __builtin_amdgcn_exp2f(x[k].x - ref) : 0.0f;
      l = fmaf(x[k].y, w, l);
      add(v[k], w);
    }
  }
  if constexpr (GROUPS > 1) {
    o_s[threadIdx.x] = o;
    if (at == 0) ml_s[threadIdx.x / LANES] = make_float2(m, l);
    __syncthreads();
    if (grp > 0 || parts == 0) return;
    const float2 *mls = ml_s + threadIdx.x / LANES;
    m = kNegInf;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) m = fmaxf(m, mls[k].x);
    l = 0.0f;
    o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      const float w = __builtin_amdgcn_exp2f(mls[k].x - (m == kNegInf ? 0.0f : m));
      l = fmaf(mls[k].y, w, l);
      add(o_s[threadIdx.x + k * LANES], w);
    }
  }
  store_four(static_cast<T *>(a.O) + row * D + 4 * at, o, l == 0.0f ? 0.0f : 1.0f / l);
  if (at == 0 && a.lse) a.lse[row] = l == 0.0f ? kNegInf : (m + __log2f(l)) * kLn2;
}

namespace {

// Key tiles that a row may see: all that the host knows of the lengths.
long most_tiles(const Args &a)
{
  return ((long)(a.window < a.cap ? a.window + kTile - 1 : a.cap) + kTile - 1) / kTile;
}
long decode_bases(const Args &a) { return (long)a.S * a.G * ((a.R + kRows - 1) / kRows); }
long decode_groups(const Args &a) { return decode_bases(a) / a.S * (a.parts ? a.parts : a.S); }

int row_bytes_of(const Args &a) { return a.d * (a.dtype == 0 ? 4 : 2); }

// Wavefronts of a decode workgroup: more of them where workgroups are few, as far as registers and keys go.
int decode_waves(const Args &a)
{
  const int most = most_decode_waves(row_bytes_of(a)), fill = fill_waves(row_bytes_of(a));
  int w = 4;
  while (w < most && decode_bases(a) * w < fill && most_tiles(a) >= 2 * w) w *= 2;
  return w;
}

}  // namespace

int decode_parts(const Args &a)
{
  const int w = decode_waves(a), fill = fill_waves(row_bytes_of(a));
  const long heads = (long)a.G * ((a.R + kRows - 1) / kRows);
  if (decode_bases(a) * w >= fill || most_tiles(a) < split_tiles(a.dtype, a.d) * w) return 0;
  if (a.S * most_tiles(a) > 1 << 22) return 0;  // (parts are counted in 32 bits and cut in fp32)
  const long parts = fill / w / heads, most = a.S * ((most_tiles(a) + 2 * w - 1) / (2 * w));
  const long n = parts < most ? parts : most;
  return (int)(n >= 2 * a.S ? n : 0);  // (no more than kMostParts: with so many tiles w is the most there is, see fits_parts)
}

namespace {

template <typename T, int D, int W>
void launch_decode_w(const Args &a, hipStream_t st)
{
  const dim3 grid((unsigned)decode_groups(a)), block(64 * W);
  // What the last-level cache cannot hold until the next token's call is not kept in the caches at all: 131071 keys 85 us so, 97 kept;
  // 74 MB 15.2 us kept, 16.4 so.
  const bool once = a.R <= kRows && (double)a.S * most_tiles(a) * kTile * a.G * D * 2 * sizeof(T) > 256e6;
  auto go = [&](auto kernel) { BLOSSOM_LAUNCH(kernel, grid, block, 0, st, a); };
  if (!a.parts) {
    if (once) go(decode_kernel<T, D, W, true, false, false>);
    else go(decode_kernel<T, D, W, false, false, false>);
    return;
  }
  if (once) go(decode_kernel<T, D, W, true, true, false>);
  else go(decode_kernel<T, D, W, false, true, false>);
  if (launch_failed()) return;
  BLOSSOM_LAUNCH((join_kernel<T, D>), dim3((unsigned)(a.S * a.H)), dim3(256), 0, st, a);
}

template <typename T, int D>
void launch_decode_d(const Args &a, hipStream_t st)
{
  constexpr int MOST = most_decode_waves(D * sizeof(T));
  const int w = decode_waves(a);
  if constexpr (MOST >= 16)
    if (w == 16) return launch_decode_w<T, D, 16>(a, st);
  if constexpr (MOST >= 8)
    if (w == 8) return launch_decode_w<T, D, 8>(a, st);
  launch_decode_w<T, D, 4>(a, st);
}

}  // namespace

bool launch_decode(const Args &a, hipStream_t st)
{
  if (!countable(decode_groups(a), 64 * decode_waves(a))) return false;
  with_type(a, [&](auto type, auto dim) { launch_decode_d<decltype(type), decltype(dim)::value>(a, st); });
  return true;
}

// Which kernel takes a prompt call, and into how many parts a row's keys go.
//  - Few 16-row tiles: their keys are shared out over the wavefronts of a workgroup each, as in decode.  That is the shortest way
//    through a walk, but every tile of keys is moved again for every 16 rows, and the fewer wavefronts a CU holds (rows of 256 bytes
//    and more), the sooner that tells.  (H = 8, G = 2, us against the other kernels, split: 500 new tokens over 1500, d = 64: 11 / 16,
//    d = 128: 16 / 20; 300 over 3700, d = 64: 17 / 18, d = 128: 28 / 24; fp32 at d = 128 200 over 4000: 64 / 53.)  Short walks go that
//    way where such workgroups are one a CU at most (172 of them, 35 new tokens over 105 for 4 sequences, fp32 at d = 128: 9.7 us / 17.8;
//    448, 16 prompts of 20 to 60, d = 64: 8.8 / 6.8).
//  - Otherwise bf16 at d = 64 or 128: 128-row workgroups on the 32x32 instructions; the rest, and sequences of 64 rows and 128 keys at
//    most, which would leave those half empty: workgroups of 32 or 64 rows (256 prompts of 16 tokens, 4 heads, d = 128: 8.8 us
//    for 11.8; of 64: 16.4 for 19.6; of 100: 31.1 for 30.7).
// Keys are split over workgroups where these do not fill the chip: up to as many as it holds at once (twice, four times as many: 54, 69
// us for 43 where 500 tokens see 10000 at d = 128), or of the small ones to eight wavefronts a SIMD, which even out ragged walks (one fp32 prompt of 8000 tokens, 2
// heads, d = 16: 211 us whole, 115, 77, 66 and 63 for 2, 4, 8 and 16 wavefronts a SIMD; 6 of 1408 to 4225, bf16, d = 8: 85 us
// whole, 85, 35, 22 and 27).  A part has 8 tiles at least (500 over 1500 at d = 64 in the 128-row kernel: 39 us whole, 20 in parts of 16
// tiles, 16 of 8, 18 of 4), and 64 where parts are many, for the join walks them one after another (16 tokens over 30000, one head,
// d = 128: 18 us in 32 parts, 20 in 64; over 131000: 36 and 30).  Walks are split from 32 tiles on (from 16: 22 us for 15 at 19 bf16 prompts
// of 168 to 505, d = 64), of the small workgroups from 24 (8 prompts of 500 to 900, 4 heads, d = 16: 19 us for 27), in fp32, whose
// tiles take longer, from 16 (4 prompts of 300 to 510, 8 heads, d = 64: 26 for 30; bf16, 30 prompts of 200 to 500, d = 32: 17 for 14).
static int shared_rows(const Args &a) { return 16 * shared_waves(row_bytes_of(a)); }
static PromptPlan prompt_plan(const Args &a)
{
  const long all = (long)a.T * a.R, tiles = most_tiles(a);
  auto groups = [&](int rows) { return (all / rows + (a.S == 1 ? (all % rows != 0) : a.S)) * a.G; };  // workgroups, nearly
  const int row_bytes = row_bytes_of(a);
  const long few = groups(kRows), most_few = row_bytes >= 512 ? 12000 : row_bytes >= 256 ? 16000 : 24000;
  PromptPlan p;
  long want;
  if (few <= 640 && few * tiles <= most_few && (few <= 256 || tiles >= 8)) {
    p.kind = kFew;
    want = 256 / few;
  } else if (prompt_mfma_supported(a) && (all > 64 * a.S || tiles > 4)) {
    p.kind = kMatrix;
    want = (a.d == 64 ? 1024 : 512) / groups(kPromptRows);
  } else {
    p.kind = kShared;
    want = 8192 / (groups(shared_rows(a)) * shared_waves(row_bytes));
  }
  const long most = tiles < (p.kind != kShared ? 32 : a.dtype == 0 ? 16 : 24) ? 1 : tiles / 64 > 32 ? tiles / 64 : tiles / 8 < 32 ? tiles / 8 : 32;
  const long n = want < most ? want : most;
  p.parts = (int)(n < 1 ? 1 : n > kMostPromptParts ? kMostPromptParts : n);
  return p;
}

int prompt_parts(const Args &a) { return prompt_plan(a).parts; }

// wavefronts of a prompt's workgroup where rows are few
static constexpr int few_waves(int row_bytes) { return most_decode_waves(row_bytes) < 8 ? most_decode_waves(row_bytes) : 8; }

bool launch_prompt(const Args &call, hipStream_t st)
{
  Args a = call;
  const PromptPlan p = prompt_plan(a);
  // (sequence s's tiles begin at floor(cu[s] R / rows) + s: enough for the last, partial one of each)
  a.row_tiles = (int)((long)a.T * a.R / (p.kind == kFew ? kRows : p.kind == kMatrix ? kPromptRows : shared_rows(a)) + a.S);
  const int waves = p.kind == kFew ? few_waves(row_bytes_of(a)) : p.kind == kMatrix ? kPromptWaves : shared_waves(row_bytes_of(a));
  if (!countable((long)a.row_tiles * a.G * a.parts, 64 * waves)) return false;
  if (p.kind == kMatrix) launch_prompt_mfma(a, st);
  else if (p.kind == kShared) launch_prompt_shared(a, st);
  with_type(a, [&](auto type, auto dim) {
    typedef decltype(type) T;
    constexpr int D = decltype(dim)::value;
    if (p.kind == kFew) {
      constexpr int W = few_waves(D * sizeof(T));
      const dim3 grid((unsigned)((long)a.row_tiles * a.G * a.parts)), block(64 * W);
      if (a.parts > 1) BLOSSOM_LAUNCH((decode_kernel<T, D, W, false, true, true>), grid, block, 0, st, a);
      else BLOSSOM_LAUNCH((decode_kernel<T, D, W, false, false, true>), grid, block, 0, st, a);
    }
    if (a.parts > 1 && !launch_failed())
      BLOSSOM_LAUNCH((join_rows_kernel<T, D>), dim3((unsigned)((size_t)a.T * a.H * (D / 4) / 256 + 1)), dim3(256), 0, st, a);
  });
  return true;
}

// Drafted trees.  Which kernel goes by the mean of a sequence's rows, for the host knows no more: sequences with one token or none count too (one
// tree of 64 tokens among 63 of one, over 4000 positions each, 32 heads over 8, d = 128: 192 us by the 16-row kernel, which walks the one
// tree's keys once for each 16 rows; that tree alone takes 41 and the others 180).  17 rows and more are the 128-row kernel's, in which
// wavefronts without rows move tiles alone (26 rows over 2000, 20000 and 131040 positions, 8 heads: 19, 26 and 92 us, the last 5.8 TB/s).
void plan_tree(Args &a)
{
  const int row_bytes = row_bytes_of(a), w = few_waves(row_bytes);
  const long rows = (long)a.T * a.R, each = rows / a.S;
  int waves, keys = kTile, least = 2 * kTreeLeast / kTile;  // workgroups that fill the chip; keys of a tile, tiles of a walk that is cut at least
  if (each <= 16) {
    // (a second launch and second pieces of walks cost as much as 9 tiles a wavefront, where they are large 5: 74 trees of one row over 1937
    // positions, d = 16, 8.7 us whole and 16.4 cut, 1 over 3205, d = 32, 12.5 and 10.3; 5 over 698, d = 128, fp32, 23.8 and 20.1)
    a.tree_rows = kRows;
    waves = fill_waves(row_bytes) / w;
    least = (row_bytes == 512 ? 5 : 9) * w;
  } else if (tree_matrix_supported(a)) {
    a.tree_rows = each <= 128 ? 128 : 256;
    waves = a.d == 64 ? 512 : 256;
    keys = 32 * 256 / a.tree_rows;
    least = 2 * kTreeLeast / keys;
  } else {
    a.tree_rows = shared_rows(a);
    waves = 4096 / shared_waves(row_bytes);
  }
  const long base = rows / a.tree_rows + a.S;  // row tiles, at most
  const long tiles = ((a.window < a.cap ? (long)a.window + kDrafts + keys - 1 : a.cap) + keys - 1) / keys;
  a.parts = waves / a.G;
  if (tiles < least || base * tiles > 1 << 30 || 3 * (rows / a.tree_rows > a.S ? rows / a.tree_rows : a.S) > 2 * a.parts) a.parts = 0;
  a.units = (int)(a.parts ? a.parts : base);
  a.slots = (int)(a.parts ? a.parts + base : 0);
}

size_t tree_part_rows(const Args &a) { return (size_t)a.slots * a.G * a.tree_rows; }

bool launch_tree(const Args &a, hipStream_t st)
{
  const bool matrix = a.tree_rows != kRows && tree_matrix_supported(a);
  // (whole walks for more than a workgroup a CU: four wavefronts where eight hold more than half a CU's LDS.  43 trees of 1 to 3 rows over 166, 8
  // heads, d = 64, bf16: 9.0 us with eight, 6.2; 103 of one row over 159 to 318, d = 32, fp32: 23.2 and 16.4; 30 of 4 to 8, d = 16, bf16: 7.8 and 8.6)
  const int few = a.parts == 0 && (long)a.units * a.G > 256 && row_bytes_of(a) >= 64 ? 4 : few_waves(row_bytes_of(a));
  const int waves = a.tree_rows == kRows ? few : matrix ? 8 : shared_waves(row_bytes_of(a));
  const dim3 grid((unsigned)((long)a.units * a.G));
  if (!countable((long)a.units * a.G, 64 * waves)) return false;
  const bool once = (double)a.S * a.cap * a.G * row_bytes_of(a) * 2 > 256e6;
  if (matrix) launch_tree_matrix(a, once, st);
  else if (a.tree_rows != kRows) launch_tree_shared(a, st);
  with_type(a, [&](auto type, auto dim) {
    typedef decltype(type) T;
    constexpr int D = decltype(dim)::value, W = few_waves(D * sizeof(T));
    if (a.tree_rows == kRows) {
      if (a.parts) BLOSSOM_LAUNCH((tree_few_kernel<T, D, W, true>), grid, dim3(64 * W), 0, st, a);
      else if (few == W) BLOSSOM_LAUNCH((tree_few_kernel<T, D, W, false>), grid, dim3(64 * W), 0, st, a);
      else BLOSSOM_LAUNCH((tree_few_kernel<T, D, 4, false>), grid, dim3(64 * 4), 0, st, a);
    }
    if (a.parts && !launch_failed()) {
      // few sequences have many parts
      constexpr int GROUPS = 256 / (D / 4) < 8 ? 256 / (D / 4) : 8;
      auto join = [&](auto kernel, int groups) {
        BLOSSOM_LAUNCH(kernel, dim3((unsigned)((size_t)a.T * a.H * groups * (D / 4) / 256 + 1)), dim3(256), 0, st, a, a.tree_rows);
      };
      if (a.parts > 8 * a.S) join(join_tree_kernel<T, D, GROUPS>, GROUPS);
      else join(join_tree_kernel<T, D, 1>, 1);
    }
  });
  return true;
}

}  // namespace paged
}  // namespace blossom
