// Prompt attention for every type and head size (bf16 at d = 64 and 128 has a kernel of its own: paged_prompt.hip).
//
// A workgroup's two wavefronts (four where a row is 256 bytes or more) take 16 rows each of one key/value head, (token, head of the
// group) pairs, and walk the 32-key tiles that any of them sees.  A tile is moved to LDS once, one step ahead, and read by all.
// Short ragged prompts are bound by the matrix pipe and the vector ALUs, which do not overlap for fp32 products (256 prompts of 20
// to 200 tokens, 2 heads, d = 32: 15.4 us, of which the products take 4.6 and the exponentials and the rest 3 at full balance).
// Tried: rings of 3, 4 and 6 tiles (23.3, 24.6, 25.4 us where 2 took 23.0), results through LDS (no gain), one wavefront a
// workgroup without barriers (as fast, slower from d = 64 on), two for large rows (d = 64 fp32: 72 us against 61).
// bf16 probabilities are rounded once, but for workgroups with rows that see few keys: both terms of them (FINE in paged_tile.h)
// everywhere take 7 to 13 % more time here (11 prompts of 3277, 3 heads over 1, d = 8: 72.4 us for 67.4; 8 of 1000 to 3000, 8 heads over
// 2, d = 32: 69.3 for 61.2), as a branch in the one walk 5 to 6 %, in a walk of their own nothing, or 0.2 of 9 us where all rows see few
// (256 prompts of 16 tokens, 4 heads, d = 128).
#include "common.h"
#include "launch.h"
#include "mfma_common.h"
#include "paged.h"
#include "paged_tile.h"

namespace blossom {
namespace paged {

using mfma::kLn2;
using mfma::kNegInf;

// wavefronts a SIMD that registers have to leave room for: bf16 at d = 128 has two registers too many by itself
template <typename T, int D>
constexpr int kRoomFor = sizeof(T) == 2 && D == 128 ? 3 : 1;

template <typename T, int D, bool SPLIT>
__global__ __launch_bounds__(64 * shared_waves(D * sizeof(T))) __attribute__((amdgpu_waves_per_eu(kRoomFor<T, D>))) void shared_kernel(Args a)
{
  typedef Tile<T, D> TL;
  constexpr int W = shared_waves(TL::RB);
  __shared__ __attribute__((aligned(1024))) char lds[2][2 * TL::BYTES];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, c = lane >> 4;

  // ---- this workgroup's rows: the last tiles, which see most keys, first ----
  const int rest = a.by_G.of(blockIdx.x), g = blockIdx.x - rest * a.G;
  const int nth = a.by_parts.of(rest), part = rest - nth * a.parts;
  const RowTile mine(a, lane, nth, 16 * W, 2);
  const int s = mine.s, tok0 = mine.tok0, new_tokens = mine.count, wg_row = mine.row0;
  if (wg_row < 0) return;
  const int rows = new_tokens * a.R;
  // (requested together: the length, the first pages, the queries)
  const int raw_len = a.kv_len[s];
  const int *table = a.page_table + s * a.table_seq;
  auto entries = [&](int first) __attribute__((always_inline)) -> int {
    const int id = table[min(first + lane, a.max_pages - 1)];
    return id >= 0 && id < a.n_pages ? id : -1;
  };
  int list0 = 0, ids = entries(0);  // pages list0 .. list0 + 63, one a lane
  const int row0 = wg_row + 16 * wv, row = row0 + n;
  const bool row_ok = row < rows;
  const int tok = a.by_R.of(row_ok ? row : rows - 1);
  const int head = g * a.R + (row_ok ? row : rows - 1) - tok * a.R;
  typename TL::Query q;
  TL::load_query(q, static_cast<const T *>(a.Q) + (tok0 + tok) * a.q_stride + (size_t)head * D, c);

  const int len = max(__builtin_amdgcn_readfirstlane(raw_len), 0);
  const int first_pos = len - new_tokens;
  const Range wg_first = seen_by(a, first_pos + a.by_R.of(wg_row), len), wg_last = seen_by(a, first_pos + a.by_R.of(min(wg_row + 16 * W, rows) - 1), len);
  const int lo = wg_first.lo, hi = wg_last.hi;  // keys that any row sees

  Range my = seen_by(a, first_pos + tok, len);
  if (!row_ok) my.hi = -1;
  // keys that all rows of the wavefront see, and that any does
  const Range r_first = seen_by(a, first_pos + a.by_R.of(min(row0, rows - 1)), len);
  const Range r_last = seen_by(a, first_pos + a.by_R.of(min(row0 + 15, rows - 1)), len);
  const int any_lo = r_first.lo, any_hi = row0 < rows ? r_last.hi : -1;

  int t = lo / kTile, t_end = hi >= lo ? hi / kTile + 1 : t;
  if constexpr (SPLIT) {
    const int each = (t_end - t + a.parts - 1) / a.parts, from = t;
    t = min(from + part * each, t_end);
    t_end = min(t + each, t_end);
  }
  const size_t page_bytes = ((size_t)a.G << a.page_shift) * TL::RB, group_bytes = ((size_t)g << a.page_shift) * TL::RB;
  // few keys: by their number, or because pages are out of range
  bool fine = TL::BF && few_keys(wg_first, wg_last);
  auto look = [&]() __attribute__((always_inline)) {
    const int page = list0 + lane;
    if (TL::BF) fine = fine || __any(ids < 0 && page >= lo >> a.page_shift && page <= hi >> a.page_shift);
  };
  look();
  auto request = [&](int t, char *to) __attribute__((always_inline)) -> unsigned {
    const int first = (t * kTile) >> a.page_shift, last = (t * kTile + kTile - 1) >> a.page_shift;
    if (first < list0 || last >= list0 + 64) {
      list0 = first;
      ids = entries(first);
      look();
    }
    const int key = t * kTile + (lane & 31);
    const int id = __shfl(ids, (key >> a.page_shift) - list0);
    const bool ok = id >= 0 && key >= lo && key <= hi;
    const unsigned seen = (unsigned)__ballot(ok);
    const size_t off = max(id, 0) * page_bytes + group_bytes + (size_t)(key & ((1 << a.page_shift) - 1)) * TL::RB;
    TL::template request<false>(a, to, to + TL::BYTES, off, ok, seen == 0xFFFFFFFFu, lane, wv, W);
    return seen;
  };

  Rows<T, D> r;
  r.clear(row_ok);
  unsigned seen = t < t_end ? request(t, lds[0]) : 0u;
#pragma unroll
  for (int i = 0; i < TL::NK; ++i) asm volatile("" : "+v"(q.x[i].x), "+v"(q.x[i].y), "+v"(q.x[i].z), "+v"(q.x[i].w));  // (arrived before the walk)
  mfma::arrived_all<0>();
  auto pair = [&](auto two) __attribute__((always_inline)) {
#pragma unroll
    for (int cur = 0; cur < 2; ++cur) {
      if (t >= t_end) break;
      const unsigned next = t + 1 < t_end ? request(t + 1, lds[cur ^ 1]) : 0u;
      const int base = t * kTile;
      if (base <= any_hi && base + kTile - 1 >= any_lo) {
        const bool all = seen == 0xFFFFFFFFu && row0 + 15 < rows && base >= r_last.lo && base + kTile - 1 <= r_first.hi;
        r.template attend<decltype(two)::value>(lds[cur], lds[cur] + TL::BYTES, q, a.scale2, seen & mfma::row_bits(my.lo - base, my.hi - base), all,
                                                base + 16 <= any_hi, lane);
      }
      mfma::arrived_all<0>();
      seen = next;
      ++t;
    }
  };
  while (t < t_end && !fine) pair(std::false_type{});
  if constexpr (TL::BF)
    while (t < t_end) pair(std::true_type{});

  const float l = r.total();
  if (!row_ok) return;
  const size_t out = (size_t)(tok0 + tok) * a.H + head;
  if constexpr (SPLIT) {
    const size_t at = out * a.parts + part;
#pragma unroll
    for (int j = 0; j < TL::NV; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (TL::channel(j, c, i) < D) a.part_o[at * D + TL::channel(j, c, i)] = r.acc[j][i];
    if (c == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(r.m, l);
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  T *O = static_cast<T *>(a.O) + out * D;
  if constexpr (TL::BF) {
#pragma unroll
    for (int j = 0; j < TL::NV; ++j)
      if (16 * j + 4 * c < D) store_four(O + 16 * j + 4 * c, make_float4(r.acc[j][0], r.acc[j][1], r.acc[j][2], r.acc[j][3]), inv);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (TL::NV >= 4) {
#pragma unroll
        for (int j = 0; j < TL::NV; j += 4)
          store_four(O + TL::channel(j, c, i), make_float4(r.acc[j][i], r.acc[j + 1][i], r.acc[j + 2][i], r.acc[j + 3][i]), inv);
      } else {
#pragma unroll
        for (int j = 0; j < TL::NV; ++j)
          if (TL::channel(j, c, i) < D) O[TL::channel(j, c, i)] = r.acc[j][i] * inv;
      }
    }
  }
  if (c == 0 && a.lse) a.lse[out] = l == 0.0f ? kNegInf : (r.m + __log2f(l)) * kLn2;
}

namespace {
template <typename T, int D>
void launch_d(const Args &a, hipStream_t st)
{
  const dim3 grid((unsigned)((long)a.row_tiles * a.G * a.parts)), block(64 * shared_waves(D * sizeof(T)));
  if (a.parts > 1) BLOSSOM_LAUNCH((shared_kernel<T, D, true>), grid, block, 0, st, a);
  else BLOSSOM_LAUNCH((shared_kernel<T, D, false>), grid, block, 0, st, a);
}
}  // namespace

void launch_prompt_shared(const Args &a, hipStream_t st)
{
  with_type(a, [&](auto type, auto dim) { launch_d<decltype(type), decltype(dim)::value>(a, st); });
}

}  // namespace paged
}  // namespace blossom
