// Attention of drafted trees on the matrix cores for bf16, d = 64 or 128, where a tree has more than 16 rows (formulas: paged_attn.hip, which
// serves fewer; other types and head sizes: paged_shared.hip).
//
// Rows are (token, head of the group) pairs of one key/value head.  A workgroup of eight wavefronts takes up to 256 of them over a share of
// their walk (TreeWork in paged.h), 32 a wavefront: RG wavefronts stand side by side for 32 RG rows, and the 8 / RG groups of them take 32
// keys of a tile each and are joined in LDS at the end, so that few rows do not leave wavefronts idle.
//  - K and V tiles go from the pages straight to LDS, once for all rows, through a ring of STAGES tiles (128 KB on a CU) with one barrier a
//    tile: a tree's rows do less with a tile than a prompt's, and memory has to be kept busy for them.
//  - S^T = K Q^T, softmax and O^T += V^T P^T as in paged_prompt.hip, but both bf16 terms of P always: P rounded to bf16 once leaves outputs off by
//    2.3e-3 of their norm where their own rounding is 1.6e-3, and trees of up to 16 rows keep both terms too.
// Measured: 26 drafted tokens over 131040 positions (32 heads over 8, d = 128: 537 MB) 129 us, 8 of it the join, where reading as many bytes
// takes 78; 33 to 64 over 4000 to 8100 for 16 sequences (412 MB, 73 GFLOP) 166 us, 10 of it the join.  The second term takes 21 and 30 of these (108
// and 136 without; 26 tokens over 131040, one head over each of 8, 92 and 89; 100 trees of 20 to 64 over 300 to 900, d = 64, 36.6 and 32.2): half as
// many matrix instructions again, and three vector instructions more a probability.  Its product after the first one's, so that the
// remainders are taken meanwhile, gains nothing.
// Of the walk with P rounded once, 136: with everything but the loads left out, 96; with the loads left out, 114; with both, 41:
// launch, finding the rows, pages and queries, 17 to 36 MB of partial sums.  Tried there: workgroups of 128 rows, two on a CU (150: K and V are moved
// twice); keys' operands read a tile ahead (no gain); the next tile's logits among this one's exponentials (145); a barrier for two tiles at
// once (139), half the wavefronts at a higher priority (no gain); 64 rows a wavefront, one a SIMD (the compiler spills).
#include "common.h"
#include "launch.h"
#include "mfma_common.h"
#include "paged.h"
#include "paged_tile.h"

namespace blossom {
namespace paged {

using mfma::bf16x8;
using mfma::f32x16;
using mfma::kLn2;
using mfma::kNegInf;
using mfma::lds_s16x4;
using mfma::s16x4;
using mfma::u32x2;

namespace {
constexpr int kWaves = 8;
}

template <int D, int RG, int STAGES, bool ONCE>
__device__ __forceinline__ void walk_tree(const Args &a, int g, const Walk &w)
{
  constexpr int KG = kWaves / RG, KEYS = 32 * KG, ROWS = 32 * RG;
  constexpr int CH = D / 8;                        // 16-byte chunks of a row
  constexpr int RPI = 64 / CH;                     // rows that a wavefront's load moves
  // A wavefront's loads of a tile: of K and of V, or, where there are fewer than wavefronts, half of these load K and half V.
  constexpr bool APART = KEYS < RPI * kWaves;
  constexpr int MOVERS = APART ? kWaves / 2 : kWaves, STEPS = KEYS / (RPI * MOVERS), LOADS = APART ? STEPS : 2 * STEPS;
  static_assert(STEPS >= 1 && STEPS * RPI * MOVERS == KEYS, "every row is moved");
  constexpr int TILE = KEYS * D;
  constexpr int NB = D / 32;                       // blocks of 32 channels
  __shared__ __attribute__((aligned(1024))) uint16_t lds[STAGES * 2 * TILE];
  __shared__ float m_s[kWaves][32], l_s[kWaves][32];
  static_assert(KG * ROWS * D * 4 <= (int)sizeof(lds), "results go where the tiles were");

  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));  // (what depends on it is not kept in registers from one walk to the next)
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rg = wv % RG, kg = wv / RG;
  const int lq = lane & 31, lh = lane >> 5;
  const int rows = w.count * a.R;
  const Tree tree(a, w.len, w.count);
  const int lo = tree.any.lo, hi = tree.any.hi;  // keys that any row sees

  // ---- this wavefront's rows; those behind the last do as it does ----
  const int row0 = w.row0 + 32 * rg, row = min(row0 + lq, rows - 1), tok = a.by_R.of(row), head = g * a.R + row - tok * a.R;
  const bool on = row0 < rows;
  const Seen sees(a, tree, a.tree[w.tok0 + tok], tok, w.count);
  bf16x8 qf[D / 16];
  {
    const uint16_t *q = static_cast<const uint16_t *>(a.Q) + (w.tok0 + tok) * a.q_stride + (size_t)head * D;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>(q + 16 * kk + 8 * lh);
  }

  // ---- the piece of the walk, and its pages: 64 entries of the list at a time, one a lane ----
  const int *table = a.page_table + w.s * a.table_seq;
  const int shift = a.page_shift;
  int t_lo = lo / KEYS, t_hi = hi >= lo ? hi / KEYS : t_lo - 1;
  t_lo = __builtin_amdgcn_readfirstlane(min(t_lo + w.from, t_hi + 1));
  t_hi = __builtin_amdgcn_readfirstlane(min(w.tiles, t_hi - t_lo + 1) + t_lo - 1);
  const int last_page = min(hi >> shift, a.max_pages - 1);
  int list0 = (t_lo * KEYS) >> shift;  // first page of the chunk
  auto entries = [&](int first) __attribute__((always_inline)) -> int {
    if (hi < lo || first + lane > last_page) return 0;  // (a page that no key of the walk needs: anything)
    const int id = table[first + lane];
    return id >= 0 && id < a.n_pages ? id : -1;
  };
  int ids = entries(list0), ids_next = entries(list0 + 64);
  unsigned long long missing;  // pages out of range
  unsigned off_lo, off_hi;     // where a page's rows of this head begin in the caches
  auto take = [&]() __attribute__((always_inline)) {
    missing = __ballot(ids < 0);
    const size_t off = (size_t)max(ids, 0) * (((size_t)a.G << shift) * (D * 2)) + ((size_t)g << shift) * (D * 2);
    off_lo = (unsigned)off;
    off_hi = (unsigned)(off >> 32);
  };
  take();
  missing &= ~0ull << max((lo >> shift) - list0, 0);  // (pages of the first tile that end before the first key: anything too)
  auto advance = [&](int page) __attribute__((always_inline)) {
    while (page >= list0 + 64) {
      list0 += 64;
      ids = ids_next;
      ids_next = entries(list0 + 64);
      take();
    }
  };

  const char *Kc = static_cast<const char *>(a.K_cache), *Vc = static_cast<const char *>(a.V_cache);
  // (the places of chunks in LDS: as in paged_prompt.hip)
  const int l_row = lane / CH, l_ch = lane % CH;
  const int mover = wv % MOVERS;
  const unsigned k_chunk = D == 128 ? (l_ch ^ ((RPI * mover + l_row) & 15)) : (l_ch ^ (((RPI * mover + l_row) >> 1) & 7));
  const unsigned v_chunk = D == 128 ? (l_ch ^ (4 * (l_row & 3))) : (l_ch ^ (2 * (l_row & 3)));
  const unsigned k_lane = l_row * (D * 2) + k_chunk * 16, v_lane = l_row * (D * 2) + v_chunk * 16;
  unsigned pages_ok = 0xFFFFFFFFu;  // lane k: of the 32 keys of this wavefront's group in the tile at place k, those that have a page
  auto request = [&](int t, int k) __attribute__((always_inline)) {
    advance((t * KEYS + KEYS - 1) >> shift);
    const unsigned to = mfma::lds_address(lds) + k * (2 * TILE * 2) + RPI * mover * (D * 2);
    const bool plain = missing == 0ull && t * KEYS >= lo && t * KEYS + KEYS - 1 <= hi;  // every row is somebody's
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int key0 = t * KEYS + RPI * (MOVERS * i + mover);
      const int at = (key0 >> shift) - list0;  // (a tile's pages lie in one chunk of the list: it begins at a tile's first page)
      const size_t off = ((size_t)(unsigned)__builtin_amdgcn_readlane(off_hi, at) << 32 | (unsigned)__builtin_amdgcn_readlane(off_lo, at)) +
                         (unsigned)((key0 & ((1 << shift) - 1)) * (D * 2));
      const char *kb = Kc + off, *vb = Vc + off;
      unsigned ko = k_lane, vo = v_lane;
      if (!plain) {
        if ((missing >> at & 1ull) != 0ull || key0 > hi || key0 + RPI - 1 < lo) {
          kb = vb = reinterpret_cast<const char *>(kZeros);
        } else {  // rows of the group that nobody sees: a seen one in their place
          const int rows_off = min(max(l_row, lo - key0), hi - key0) - l_row;
          ko += rows_off * (D * 2);
          vo += rows_off * (D * 2);
        }
      }
      if (!APART || wv < MOVERS) to_lds<ONCE>(kb, ko, to + i * (RPI * MOVERS * D * 2));
      if (!APART || wv >= MOVERS) to_lds<ONCE>(vb, vo, to + TILE * 2 + i * (RPI * MOVERS * D * 2));
    }
    unsigned ok = 0xFFFFFFFFu;
    if (missing != 0ull) {
      ok = 0u;
      for (int j = 0; j < 32; j += 8)
        if ((missing >> ((((t * KEYS + 32 * kg + j) >> shift) - list0) & 63) & 1ull) == 0ull) ok |= 0xFFu << j;
    }
    pages_ok = lane == k ? ok : pages_ok;
  };

  // ---- LDS read offsets (elements), of this wavefront's 32 keys ----
  int koff[D / 16];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk)
    koff[kk] = (32 * kg + lq) * D + (((2 * kk + lh) ^ (D == 128 ? lq & 15 : (lq >> 1) & 7)) * 8);
  const int r16 = lane & 15;
  int voff[NB];
#pragma unroll
  for (int mb = 0; mb < NB; ++mb)
    voff[mb] = TILE + (32 * kg + 4 * lh + (r16 >> 2)) * D +
               (((4 * mb + 2 * ((lane >> 4) & 1) + ((r16 & 3) >> 1)) ^ ((D == 128 ? 4 : 2) * (r16 >> 2))) * 8) + 4 * (r16 & 1);

  f32x16 oacc[NB];
#pragma unroll
  for (int mb = 0; mb < NB; ++mb)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[mb][i] = 0.0f;
  float ref = 0.0f, l_run = 0.0f;
  bool fresh = true;  // no visible key met yet
  // raises the reference to the row's maximum of this tile, or places it
  auto move_ref = [&](const f32x16 &sc) __attribute__((always_inline)) {
    float mx = sc[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
    const u32x2 sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * a.scale2;
    const bool up = mx != kNegInf && (fresh || mx > ref);
    const float to = up ? mx : ref;
    const float f = up && !fresh ? __builtin_amdgcn_exp2f(ref - to) : 1.0f;
    l_run *= f;
#pragma unroll
    for (int mb = 0; mb < NB; ++mb)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[mb][i] *= f;
    ref = to;
    fresh = fresh && !up;
  };

  // ---- the walk ----
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) asm volatile("" : "+v"(qf[kk]));  // (arrived before the first request)
  asm volatile("" : "+v"(ids_next));
#pragma unroll 1
  for (int k = 0; k < STAGES - 1; ++k)
    if (t_lo + k <= t_hi) request(t_lo + k, k);
  int t = t_lo, k = 0;
#pragma unroll 1
  while (t <= t_hi) {
    // when a tile has arrived, everybody is done with the one before it, whose place the next request takes
    if (t + STAGES - 2 <= t_hi) mfma::arrived_all<LOADS *(STAGES - 2)>();
    else mfma::arrived_all<0>();
    const int here = k, base = t * KEYS + 32 * kg;
    if (t + STAGES - 1 <= t_hi) request(t + STAGES - 1, k == 0 ? STAGES - 1 : k - 1);
    k = k == STAGES - 1 ? 0 : k + 1;
    ++t;
    if (!on) continue;
    const uint16_t *ks = lds + here * (2 * TILE);
    bf16x8 kf[D / 16], vf[2][NB];
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) kf[kk] = *reinterpret_cast<const bf16x8 *>(ks + koff[kk]);
    __builtin_amdgcn_sched_barrier(0);  // keys' operands are requested together, values' between the products
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int mb = 0; mb < NB; ++mb) {
        const uint16_t *v0 = ks + 16 * h * D + voff[mb];
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(v0));
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(v0 + 8 * D));
        vf[h][mb] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    f32x16 sc;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], qf[kk], sc, 0, 0, 0);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    const unsigned ok = (unsigned)__builtin_amdgcn_readlane(pages_ok, here);
    if (base < tree.every.lo || base + 31 > tree.every.hi || ok != 0xFFFFFFFFu)
      mfma::keep_rows(sc, sees.bits(tree, base, mfma::row_bits) & ok, lh, kNegInf);
    bf16x8 pf[2], rest[2];
    float sum, scale = a.scale2;
    bool placed = __any(fresh || is_far(ref));
#pragma unroll 1
    for (;;) {
      if (placed) {
        move_ref(sc);
        if (__any(is_far(ref))) {
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[i] = rounded_product(sc[i], a.scale2);
          scale = 1.0f;
        }
      }
      float sa, sb;
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float pa = __builtin_amdgcn_exp2f(fmaf(sc[i], scale, -ref));
        const float pb = __builtin_amdgcn_exp2f(fmaf(sc[i + 1], scale, -ref));
        pf[i >> 3][i & 7] = (__bf16)pa;
        pf[i >> 3][(i & 7) + 1] = (__bf16)pb;
        rest[i >> 3][i & 7] = (__bf16)(pa - (float)pf[i >> 3][i & 7]);
        rest[i >> 3][(i & 7) + 1] = (__bf16)(pb - (float)pf[i >> 3][(i & 7) + 1]);
        sa = i == 0 ? pa : sa + pa;
        sb = i == 0 ? pb : sb + pb;
      }
      sum = sa + sb;
      if (placed || !__any(!(sum <= kSumLimit))) break;
      placed = true;
    }
    l_run += sum;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int mb = 0; mb < NB; ++mb) {
        oacc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[h][mb], rest[h], oacc[mb], 0, 0, 0);
        oacc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[h][mb], pf[h], oacc[mb], 0, 0, 0);
      }
  }
  mfma::arrived_all<0>();

  // ---- results: through LDS, where the key groups are joined and neighbouring lanes get neighbouring channels.  Chunk c (16 bytes) of a row
  // at c ^ (the row modulo a row's chunks) ----
  float *out_s = reinterpret_cast<float *>(lds);
  if (on) {
    const float l = l_run + __shfl_xor(l_run, 32);
    const int r = 32 * rg + lq;
    if (lh == 0) {
      m_s[wv][lq] = l == 0.0f ? kNegInf : ref;
      l_s[wv][lq] = l;
    }
#pragma unroll
    for (int mb = 0; mb < NB; ++mb)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4 *>(out_s + ((size_t)(kg * ROWS + r) * (D / 4) + ((8 * mb + 2 * q + lh) ^ (r & (D / 4 - 1)))) * 4) =
            make_float4(oacc[mb][4 * q], oacc[mb][4 * q + 1], oacc[mb][4 * q + 2], oacc[mb][4 * q + 3]);
  }
  __syncthreads();
  const int here = min(rows - w.row0, ROWS);
  for (int e = threadIdx.x; e < here * (D / 4); e += 64 * kWaves) {
    const int r = e / (D / 4), c = e % (D / 4), side = r / 32, in = r % 32;
    float mm = kNegInf;
#pragma unroll
    for (int j = 0; j < KG; ++j) mm = fmaxf(mm, m_s[j * RG + side][in]);
    const float to = mm == kNegInf ? 0.0f : mm;
    float ll = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < KG; ++j) {
      const float f = __builtin_amdgcn_exp2f(m_s[j * RG + side][in] - to);
      const float4 v = *reinterpret_cast<const float4 *>(out_s + ((size_t)(j * ROWS + r) * (D / 4) + (c ^ (r & (D / 4 - 1)))) * 4);
      ll = fmaf(l_s[j * RG + side][in], f, ll);
      o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
    }
    if (w.slot >= 0) {
      const size_t at = ((size_t)w.slot * a.G + g) * ROWS + r;
      *reinterpret_cast<float4 *>(a.part_o + at * D + 4 * c) = o;
      if (c == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(mm, ll);
    } else {
      const int tok = a.by_R.of(w.row0 + r);
      const size_t out = (size_t)(w.tok0 + tok) * a.H + g * a.R + w.row0 + r - tok * a.R;
      store_four(static_cast<bf16_t *>(a.O) + out * D + 4 * c, o, ll == 0.0f ? 0.0f : 1.0f / ll);
      if (c == 0 && a.lse) a.lse[out] = ll == 0.0f ? kNegInf : (mm + __log2f(ll)) * kLn2;
    }
  }
}

template <int D, int RG, int STAGES, int EU, bool ONCE>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(EU, EU))) void tree_kernel(Args a)
{
  const int lane = threadIdx.x & 63, block = tree_block(a), rest = a.by_G.of(block), g = block - rest * a.G;
  constexpr int KEYS = 32 * kWaves / RG;
  TreeWork work(rest, 32 * RG, KEYS);
  for (Walk w = work.begin(a, lane, kTreeLeast / KEYS); w.s >= 0; w = work.next(a, lane)) {
    work.tell(a, w, g, lane, threadIdx.x, 64 * kWaves);
    walk_tree<D, RG, STAGES, ONCE>(a, g, w);
    __syncthreads();
  }
}

bool tree_matrix_supported(const Args &a) { return a.dtype == 1 && (a.d == 64 || a.d == 128); }

void launch_tree_matrix(const Args &a, bool once, hipStream_t st)
{
  auto go = [&](auto kernel) { BLOSSOM_LAUNCH(kernel, dim3((unsigned)((long)a.units * a.G)), dim3(64 * kWaves), 0, st, a); };
  auto pick = [&](auto past) {
    constexpr bool ONCE = decltype(past)::value;
    if (a.d == 128) {
      if (a.tree_rows == 256) go(tree_kernel<128, 8, 8, 2, ONCE>);
      else go(tree_kernel<128, 4, 4, 2, ONCE>);
    } else {
      if (a.tree_rows == 256) go(tree_kernel<64, 8, 8, 4, ONCE>);
      else go(tree_kernel<64, 4, 4, 4, ONCE>);
    }
  };
  if (once) pick(std::true_type{});
  else pick(std::false_type{});
}

}  // namespace paged
}  // namespace blossom
