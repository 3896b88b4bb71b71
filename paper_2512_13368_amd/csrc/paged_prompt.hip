// Prompt attention on the matrix cores for bf16, d = 64 or 128 (formulas: paged_attn.hip, which serves everything else).
//
// A workgroup of four wavefronts takes 128 query rows of one key/value head, 32 a wavefront, and walks the 64-key tiles that any of
// them sees.  Rows are (token, head of the group) pairs, R = H/G of them a token, so that heads that share keys share the tiles too
// and a short prompt fills its workgroups.  K and V tiles go from the pages straight to LDS (eight or four rows an instruction: always
// of one page), one tile ahead or two; every wavefront reads them whole.
//  - S^T = K Q^T on v_mfma_f32_32x32x16_bf16: a lane owns one query row and 16 of a half tile's 32 logits.
//  - softmax in fp32, base 2: p = exp2(scale2 * s - ref).  The reference is a row's maximum over the first keys it meets; it is
//    raised only when a lane's probabilities of a half tile pass 4096 in sum, so the usual half tile takes no maximum (one far from 0
//    does: see kFar in paged.h).
//  - O^T += V^T P^T with P^T straight from the accumulator registers (rounded to bf16, as the matrix instruction wants them; the
//    sum is of the unrounded ones) and V^T through the transposing LDS read.  What the rounding leaves of P is a second product in
//    workgroups with rows that see few keys, which have a walk of their own (as a branch in the one walk it takes 1.3 to 1.6 % of long
//    prompts).  Everywhere, as in decode, the error in norm falls from 2.2e-3 to 1.6e-3, for a third more time (long prompts 1075 us for
//    795, chunks 175 for 128, ragged ones 160 for 121): not taken.
//
// Measured under steady load: two prompts of 6001 and 8191 tokens, 32 heads over 8, d = 128: 815 us, 1.04 PFLOP/s, where a bf16 product
// of 8192^3 reaches 1.07; chunks of 512 over a window of 4096: 131 us, 870 TFLOP/s; 32 ragged prompts of 7 to 1997, 16 heads over 4,
// d = 64: 124 us, 720 TFLOP/s.  (Other cards: 797 to 850 us for the long ones, one 949.  In the first milliseconds after a pause the card's clock dips: 884, 1053 and 851 us at the first, fifth
// and twentieth of the long calls.)  The matrix pipe is busy 52 % (d = 64: 41 %) and the vector ALUs' issue port 46 % (75 %) of the
// time: a half tile's 16 exponentials alone are 256 cycles beside 512 (256) of products, and the two overlap in part.  Tried: both halves' logits
// before the exponentials (848 against 836 us, 137 against 134 and 129), three wavefronts a SIMD instead of four at d = 64 (154 us
// against 143 at the time).
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

constexpr int kWaves = kPromptWaves;
constexpr int kKeys = 64;                  // keys of a tile
}  // namespace

template <int D, int STAGES, int WAVES_EU>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(WAVES_EU, WAVES_EU))) void prompt_kernel(Args a)
{
  constexpr int CH = D / 8;              // 16-byte chunks of a row
  constexpr int RPI = 64 / CH;           // rows that a wavefront's load moves
  constexpr int LOADS = kKeys / (RPI * kWaves);  // such loads of K a wavefront and tile (and as many of V)
  constexpr int TILE = kKeys * D;
  constexpr int NB = D / 32;             // blocks of 32 channels
  __shared__ __attribute__((aligned(1024))) uint16_t lds[2 * STAGES * TILE];
  uint16_t(*Ks)[TILE] = reinterpret_cast<uint16_t(*)[TILE]>(lds), (*Vs)[TILE] = Ks + STAGES;

  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lq = lane & 31, lh = lane >> 5;

  // ---- this workgroup's rows: the last tiles, which see most keys, first ----
  const int rest = a.by_G.of(blockIdx.x), g = blockIdx.x - rest * a.G;
  const int nth = a.by_parts.of(rest), part = rest - nth * a.parts;
  const RowTile mine(a, lane, nth, kPromptRows, 8);
  const int s = mine.s, tok0 = mine.tok0, new_tokens = mine.count, wg_row = mine.row0;
  if (wg_row < 0) return;
  const int rows = new_tokens * a.R;
  const int len = max(__builtin_amdgcn_readfirstlane(a.kv_len[s]), 0);
  const int first_pos = len - new_tokens;

  const Range all_first = seen_by(a, first_pos + a.by_R.of(wg_row), len);
  const Range all_last = seen_by(a, first_pos + a.by_R.of(min(wg_row + kPromptRows, rows) - 1), len);
  const int lo = all_first.lo, hi = all_last.hi;  // keys that any row of the workgroup sees

  const int row0 = wg_row + 32 * wv, row = row0 + lq;
  const bool row_ok = row < rows;
  const int tok = a.by_R.of(row_ok ? row : rows - 1);
  const int head = g * a.R + (row_ok ? row : rows - 1) - tok * a.R;
  Range my = seen_by(a, first_pos + tok, len);
  if (!row_ok) my.hi = -1;
  // keys that all rows of the wavefront see, and that any does (rows ascend with positions)
  const bool wave_on = row0 < rows;
  const int w_first = first_pos + a.by_R.of(min(row0, rows - 1)), w_last = first_pos + a.by_R.of(min(row0 + 31, rows - 1));
  const Range r_first = seen_by(a, w_first, len), r_last = seen_by(a, w_last, len);
  const int every_lo = row0 + 31 < rows ? r_last.lo : 0x7FFFFFFF, every_hi = r_first.hi;
  const int any_lo = r_first.lo, any_hi = wave_on ? r_last.hi : -1;

  bf16x8 qf[D / 16];
  {
    const uint16_t *q = static_cast<const uint16_t *>(a.Q) + (tok0 + tok) * a.q_stride + (size_t)head * D;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *reinterpret_cast<const bf16x8 *>(q + 16 * kk + 8 * lh);
  }

  // ---- page list: 64 entries at a time, one a lane ----
  const int *table = a.page_table + s * a.table_seq + g * a.table_group;
  const int shift = a.page_shift;
  int t_lo = lo / kKeys, t_hi = hi >= lo ? hi / kKeys : t_lo - 1;
  if (a.parts > 1) {
    const int each = (t_hi - t_lo + a.parts) / a.parts, from = t_lo;
    t_lo = __builtin_amdgcn_readfirstlane(min(from + part * each, t_hi + 1));
    t_hi = __builtin_amdgcn_readfirstlane(min(t_lo + each - 1, t_hi));
  }
  const int last_page = min(hi >> shift, a.max_pages - 1);
  int list0 = (t_lo * kKeys) >> shift;  // first page of the chunk
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
  bool fine = few_keys(all_first, all_last) || missing != 0ull;  // few keys: by their number, or because pages are out of range
  auto advance = [&](int page) __attribute__((always_inline)) {
    while (page >= list0 + 64) {
      list0 += 64;
      ids = ids_next;
      ids_next = entries(list0 + 64);
      take();
      fine = fine || missing != 0ull;
    }
  };

  const char *Kc = static_cast<const char *>(a.K_cache), *Vc = static_cast<const char *>(a.V_cache);
  // LDS position of chunk c of row r: c ^ swz(r); K: its low bits of r or of r / 2, V: (r & 3) blocks of 64 or 32 bytes: both the
  // row-per-lane 16-byte reads and the transposing reads of four rows then meet every bank once
  const int l_row = lane / CH, l_ch = lane % CH;
  const unsigned k_chunk = D == 128 ? (l_ch ^ ((RPI * wv + l_row) & 15)) : (l_ch ^ (((RPI * wv + l_row) >> 1) & 7));
  const unsigned v_chunk = D == 128 ? (l_ch ^ (4 * (l_row & 3))) : (l_ch ^ (2 * (l_row & 3)));
  const unsigned k_lane = l_row * (D * 2) + k_chunk * 16, v_lane = l_row * (D * 2) + v_chunk * 16;

  auto stage = [&](int t, uint16_t *ks, uint16_t *vs) __attribute__((always_inline)) {
    advance((t * kKeys + kKeys - 1) >> shift);
    const unsigned k_to = mfma::lds_address(ks) + RPI * wv * (D * 2), v_to = mfma::lds_address(vs) + RPI * wv * (D * 2);
    const bool plain = missing == 0ull && t * kKeys >= lo && t * kKeys + kKeys - 1 <= hi;  // every row is somebody's
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int key0 = t * kKeys + RPI * (kWaves * i + wv);
      const int at = (key0 >> shift) - list0;  // (a tile's pages lie in one chunk of the list: pages of 8 make a tile of 8)
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
      to_lds<false>(kb, ko, k_to + i * (RPI * kWaves * D * 2));
      to_lds<false>(vb, vo, v_to + i * (RPI * kWaves * D * 2));
    }
  };

  // ---- LDS read offsets (elements) ----
  int koff[D / 16];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk)
    koff[kk] = lq * D + (((2 * kk + lh) ^ (D == 128 ? lq & 15 : (lq >> 1) & 7)) * 8);
  const int r16 = lane & 15;
  int voff[NB];
#pragma unroll
  for (int mb = 0; mb < NB; ++mb)
    voff[mb] = (4 * lh + (r16 >> 2)) * D +
               (((4 * mb + 2 * ((lane >> 4) & 1) + ((r16 & 3) >> 1)) ^ ((D == 128 ? 4 : 2) * (r16 >> 2))) * 8) + 4 * (r16 & 1);

  f32x16 oacc[NB];
#pragma unroll
  for (int mb = 0; mb < NB; ++mb)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[mb][i] = 0.0f;
  float ref = 0.0f, l_run = 0.0f;
  bool fresh = row_ok;  // no visible key met yet

  // raises the reference to the row's maximum of this half tile, or places it
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

  auto half = [&](const uint16_t *ks, const uint16_t *vs, int base, unsigned pages_ok, auto two) __attribute__((always_inline)) {
    if (base > any_hi || base + 31 < any_lo) return;
    bf16x8 kf[D / 16];
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) kf[kk] = *reinterpret_cast<const bf16x8 *>(ks + koff[kk]);
    __builtin_amdgcn_sched_barrier(0);  // keys' operands are requested together, values' between the products
    bf16x8 vf[2][NB];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int mb = 0; mb < NB; ++mb) {
        const uint16_t *v0 = vs + 16 * t * D + voff[mb];
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(v0));
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(v0 + 8 * D));
        vf[t][mb] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
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
    if (base < every_lo || base + 31 > every_hi || pages_ok != 0xFFFFFFFFu)
      mfma::keep_rows(sc, mfma::row_bits(my.lo - base, my.hi - base) & pages_ok, lh, kNegInf);
    constexpr bool TWO = decltype(two)::value;
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
        if constexpr (TWO) {
          rest[i >> 3][i & 7] = (__bf16)(pa - (float)pf[i >> 3][i & 7]);
          rest[i >> 3][(i & 7) + 1] = (__bf16)(pb - (float)pf[i >> 3][(i & 7) + 1]);
        }
        sa = i == 0 ? pa : sa + pa;
        sb = i == 0 ? pb : sb + pb;
      }
      sum = sa + sb;
      if (placed || !__any(!(sum <= kSumLimit))) break;
      placed = true;
    }
    l_run += sum;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int mb = 0; mb < NB; ++mb) {
        if constexpr (TWO) oacc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t][mb], rest[t], oacc[mb], 0, 0, 0);
        oacc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t][mb], pf[t], oacc[mb], 0, 0, 0);
      }
  };

  // bit k: key base + k has a page
  auto pages_of = [&](int base) __attribute__((always_inline)) -> unsigned {
    unsigned bits = 0u;
    for (int k = 0; k < 32; k += 8)
      if ((missing >> ((((base + k) >> shift) - list0) & 63) & 1ull) == 0ull) bits |= 0xFFu << k;
    return bits;
  };

  // ---- the walk ----
  if (t_hi >= t_lo) stage(t_lo, Ks[0], Vs[0]);
  // (the compiler has the queries arrive here: it would wait for them in the loop, and for the tiles on their way with them)
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) asm volatile("" : "+v"(qf[kk]));
  asm volatile("" : "+v"(ids_next));
  mfma::arrived_all<0>();
  auto step = [&](int t, auto buffer, auto two) __attribute__((always_inline)) {
    constexpr int cur = decltype(buffer)::value;
    unsigned ok0 = 0xFFFFFFFFu, ok1 = 0xFFFFFFFFu;
    if (missing != 0ull) {  // (before the list moves on)
      ok0 = pages_of(t * kKeys);
      ok1 = pages_of(t * kKeys + 32);
    }
    if (t < t_hi) stage(t + 1, Ks[cur ^ 1], Vs[cur ^ 1]);
    half(Ks[cur], Vs[cur], t * kKeys, ok0, two);
    half(Ks[cur] + 32 * D, Vs[cur] + 32 * D, t * kKeys + 32, ok1, two);
    mfma::arrived_all<0>();
  };
  int t = t_lo;
  for (; t <= t_hi && !fine; t += 2) {
    step(t, std::integral_constant<int, 0>{}, std::false_type{});
    if (t < t_hi) step(t + 1, std::integral_constant<int, 1>{}, std::false_type{});
  }
  for (; t <= t_hi; t += 2) {
    step(t, std::integral_constant<int, 0>{}, std::true_type{});
    if (t < t_hi) step(t + 1, std::integral_constant<int, 1>{}, std::true_type{});
  }

  // ---- results ----
  l_run += __shfl_xor(l_run, 32);
  const size_t out = (size_t)(tok0 + tok) * a.H + head;
  if (a.parts > 1) {  // sums as they are, for the join
    if (!row_ok) return;
    const size_t at = out * a.parts + part;
#pragma unroll
    for (int mb = 0; mb < NB; ++mb)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4 *>(a.part_o + at * D + 32 * mb + 8 * q + 4 * lh) =
            make_float4(oacc[mb][4 * q], oacc[mb][4 * q + 1], oacc[mb][4 * q + 2], oacc[mb][4 * q + 3]);
    if (lh == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(l_run == 0.0f ? kNegInf : ref, l_run);
    return;
  }
  // A lane holds pieces of a row: they go through LDS, where the tiles were, so that neighbouring lanes store neighbouring bytes.
  // Chunk c of row r at c ^ (r modulo a row's chunks).
  const float inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;
  char *mine_out = reinterpret_cast<char *>(lds) + wv * (32 * D * 2);
#pragma unroll
  for (int mb = 0; mb < NB; ++mb)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<uint2 *>(mine_out + lq * (D * 2) + (((4 * mb + q) ^ (lq & (CH - 1))) * 16) + 8 * lh) =
          make_uint2(mfma::pack2_bf16(oacc[mb][4 * q] * inv, oacc[mb][4 * q + 1] * inv), mfma::pack2_bf16(oacc[mb][4 * q + 2] * inv, oacc[mb][4 * q + 3] * inv));
  if (row_ok && lh == 0 && a.lse) a.lse[out] = l_run == 0.0f ? kNegInf : (ref + __log2f(l_run)) * kLn2;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (a wavefront reads what it wrote itself)
#pragma unroll
  for (int i = 0; i < 32 / RPI; ++i) {
    const int r = RPI * i + l_row;
    if (row0 + r >= rows) continue;
    const uint4 x = *reinterpret_cast<const uint4 *>(mine_out + r * (D * 2) + ((l_ch ^ (r & (CH - 1))) * 16));
    const int tk = a.by_R.of(row0 + r);
    *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.O) + ((size_t)(tok0 + tk) * a.H + g * a.R + row0 + r - tk * a.R) * D + 8 * l_ch) = x;
  }
}

bool prompt_mfma_supported(const Args &a) { return a.dtype == 1 && (a.d == 64 || a.d == 128); }

void launch_prompt_mfma(const Args &a, hipStream_t st)
{
  const dim3 grid((unsigned)((long)a.row_tiles * a.G * a.parts)), block(64 * kWaves);
  if (a.d == 64) BLOSSOM_LAUNCH((prompt_kernel<64, 2, 4>), grid, block, 0, st, a);
  else BLOSSOM_LAUNCH((prompt_kernel<128, 2, 2>), grid, block, 0, st, a);
}

}  // namespace paged
}  // namespace blossom
