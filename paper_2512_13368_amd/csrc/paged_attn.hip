// Attention over a paged key/value cache: one new token a sequence (decode), or a run of new tokens (prompt).
//
//   o = sum_j p_j V_j,  p = softmax_j(scale q.K_j)   over the cached positions j that the query sees:
//   j <= pos, pos - j < window, pos = kv_len - new + i for new token i (decode: pos = kv_len - 1)
//
// Query rows are (token, head) pairs that share a key/value head: R = H/G heads of a token read the same keys, so a wavefront
// takes 16 such rows and 32 keys a step, on 16x16 matrix instructions, with operands straight from memory to registers:
//  - S^T = K Q^T: a lane's 16 bytes of a key row are an operand as they are.  The result leaves lane (row n, group c) with the
//    logits of keys 16t + 4c + i (t < 2, i < 4).
//  - O^T += V^T P^T: the sum over keys may run in any order, so lane group c takes the keys whose probabilities it holds, and P^T
//    is an operand as it is.  V^T wants 8 keys of one channel in a lane: it loads d/16 channels of its 8 keys and turns that block
//    in its registers (bf16; fp32 needs no turn).  A lane then holds channels of its own row, so the running maximum and sum
//    (fp32, log2 units) need no exchange for the rescaling.
// Four wavefronts of a workgroup take a row tile's key tiles in turn and join their results in LDS; where rows are few, a row's
// keys are split over workgroups too, whose sums another kernel joins.
#include "common.h"
#include "launch.h"
#include "mfma_common.h"
#include "paged.h"

namespace blossom {
namespace paged {

namespace {

using mfma::bf16x8;
using mfma::kLn2;
using mfma::kNegInf;
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kRows = 16;   // query rows of a workgroup
constexpr int kTile = 32;   // keys of a step
constexpr int kWaves = 4;
constexpr int kMostSplits = 256;

// Operands of one step in registers, by storage type and head size.
template <typename T, int D>
struct Ops;

template <int D>
struct Ops<bf16_t, D> {
  static constexpr int NK = D >= 32 ? D / 32 : 1;  // matrix instructions for 16 keys' logits
  static constexpr int VPT = D >= 16 ? D / 16 : 1; // channels of V in a lane
  uint4 q[NK], k[2][NK];
  uint32_t v[8][VPT >= 2 ? VPT / 2 : 1];
  // d < 32: channels beyond the row are zeros
  static __device__ __forceinline__ void row(uint4 (&to)[NK], const bf16_t *p, int c)
  {
    if constexpr (D >= 32) {
#pragma unroll
      for (int i = 0; i < NK; ++i) to[i] = *reinterpret_cast<const uint4 *>(p + 32 * i + 8 * c);
    } else {
      to[0] = make_uint4(0, 0, 0, 0);
      if (8 * c < D) to[0] = *reinterpret_cast<const uint4 *>(p + 8 * c);
    }
  }
  __device__ __forceinline__ void load_v(int slot, const bf16_t *p, int m)
  {
    if constexpr (VPT == 8) {
      const uint4 x = *reinterpret_cast<const uint4 *>(p + 8 * m);
      v[slot][0] = x.x; v[slot][1] = x.y; v[slot][2] = x.z; v[slot][3] = x.w;
    } else if constexpr (VPT == 4) {
      const uint2 x = *reinterpret_cast<const uint2 *>(p + 4 * m);
      v[slot][0] = x.x; v[slot][1] = x.y;
    } else if constexpr (VPT == 2) {
      v[slot][0] = *reinterpret_cast<const uint32_t *>(p + 2 * m);
    } else {
      v[slot][0] = m < D ? (uint32_t)p[m].bits : 0u;
    }
  }
  __device__ __forceinline__ void clear_v(int slot)
  {
#pragma unroll
    for (int i = 0; i < (VPT >= 2 ? VPT / 2 : 1); ++i) v[slot][i] = 0u;
  }
  __device__ __forceinline__ f32x4 logits(int t) const
  {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NK; ++i)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][i]), __builtin_bit_cast(bf16x8, q[i]), s, 0, 0, 0);
    return s;
  }
  // The probabilities are rounded to bf16, as the matrix instruction wants them; their sum is of the unrounded ones.
  __device__ __forceinline__ void product(const float (&p)[8], f32x4 (&acc)[VPT]) const
  {
    bf16x8 pf;
#pragma unroll
    for (int i = 0; i < 8; ++i) pf[i] = (__bf16)p[i];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
      const uint4 vt = make_uint4(w[0], w[1], w[2], w[3]);
      acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt), __builtin_bit_cast(bf16x8, pf), acc[j], 0, 0, 0);
    }
  }
};

template <int D>
struct Ops<float, D> {
  static constexpr int NK = D >= 16 ? D / 16 : 1;
  static constexpr int VPT = D >= 16 ? D / 16 : 1;
  float4 q[NK], k[2][NK];
  float v[8][VPT];
  static __device__ __forceinline__ void row(float4 (&to)[NK], const float *p, int c)
  {
    if constexpr (D >= 16) {
#pragma unroll
      for (int i = 0; i < NK; ++i) to[i] = *reinterpret_cast<const float4 *>(p + 16 * i + 4 * c);
    } else {
      to[0] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (4 * c < D) to[0] = *reinterpret_cast<const float4 *>(p + 4 * c);
    }
  }
  __device__ __forceinline__ void load_v(int slot, const float *p, int m)
  {
    if constexpr (VPT >= 4) {
#pragma unroll
      for (int j = 0; j < VPT; j += 4) {
        const float4 x = *reinterpret_cast<const float4 *>(p + VPT * m + j);
        v[slot][j] = x.x; v[slot][j + 1] = x.y; v[slot][j + 2] = x.z; v[slot][j + 3] = x.w;
      }
    } else if constexpr (VPT == 2) {
      const float2 x = *reinterpret_cast<const float2 *>(p + 2 * m);
      v[slot][0] = x.x; v[slot][1] = x.y;
    } else {
      v[slot][0] = m < D ? p[m] : 0.0f;
    }
  }
  __device__ __forceinline__ void clear_v(int slot)
  {
#pragma unroll
    for (int i = 0; i < VPT; ++i) v[slot][i] = 0.0f;
  }
  __device__ __forceinline__ f32x4 logits(int t) const
  {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][i].x, q[i].x, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][i].y, q[i].y, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][i].z, q[i].z, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][i].w, q[i].w, s, 0, 0, 0);
    }
    return s;
  }
  __device__ __forceinline__ void product(const float (&p)[8], f32x4 (&acc)[VPT]) const
  {
#pragma unroll
    for (int slot = 0; slot < 8; ++slot)
#pragma unroll
      for (int j = 0; j < VPT; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[slot][j], p[slot], acc[j], 0, 0, 0);
  }
};

__device__ __forceinline__ void store_out(float *p, float x) { *p = x; }
__device__ __forceinline__ void store_out(bf16_t *p, float x) { p->bits = __builtin_bit_cast(uint16_t, (__bf16)x); }

}  // namespace

template <typename T, int D, bool PROMPT>
__global__ __launch_bounds__(64 * kWaves) void rows_kernel(Args a)
{
  typedef Ops<T, D> O_;
  constexpr int VPT = O_::VPT;
  constexpr int LDR = D + 4;  // floats of an LDS row
  __shared__ __attribute__((aligned(16))) float acc_s[kWaves][kRows][LDR];
  __shared__ float m_s[kWaves][kRows], l_s[kWaves][kRows];

  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, c = lane >> 4;

  // ---- this workgroup's rows ----
  const unsigned g = blockIdx.x % a.G;
  const unsigned rest = blockIdx.x / a.G;
  const int split = (int)(rest % a.nsplit);
  const int tile = (int)(rest / a.nsplit);
  int s, row0, rows, tok0, new_tokens;
  if constexpr (PROMPT) {
    s = find_sequence(a.S, lane, [&](int i) { return (int)((long)token_at(a, i) * a.R / kRows) + i <= tile; });
    tok0 = token_at(a, s);
    new_tokens = max(token_at(a, s + 1) - tok0, 0);
    row0 = (tile - (int)((long)tok0 * a.R / kRows) - s) * kRows;
    rows = new_tokens * a.R;  // (T * R fits 31 bits: checked at the boundary)
  } else {
    const int tiles = (a.R + kRows - 1) / kRows;
    s = tile / tiles;
    tok0 = s;
    new_tokens = 1;
    row0 = (tile % tiles) * kRows;
    rows = a.R;
  }
  if (row0 >= rows || row0 < 0) return;
  const int len = max(a.kv_len[s], 0);
  const int first_pos = len - new_tokens;

  const int row = row0 + n;
  const bool row_ok = row < rows;
  const int tok = PROMPT ? (row_ok ? row : rows - 1) / a.R : 0;
  const int head = g * a.R + (row_ok ? row : rows - 1) - tok * a.R;
  Range my = seen_by(a, first_pos + tok, len);
  if (!row_ok) my.hi = -1;
  int lo, hi;  // of all rows together
  if constexpr (PROMPT) {
    lo = seen_by(a, first_pos + row0 / a.R, len).lo;
    hi = seen_by(a, first_pos + (min(row0 + kRows, rows) - 1) / a.R, len).hi;
  } else {
    lo = seen_by(a, first_pos, len).lo;
    hi = seen_by(a, first_pos, len).hi;
  }

  O_ x;
  {
    const T *q = static_cast<const T *>(a.Q) + (tok0 + tok) * a.q_stride + (size_t)head * D;
    O_::row(x.q, q, c);
  }

  // ---- key tiles of this part ----
  const int t_lo = lo / kTile, t_all = hi >= lo ? hi / kTile - t_lo + 1 : 0;
  const int chunk = max((t_all + a.nsplit - 1) / a.nsplit, kWaves);
  const int t_begin = t_lo + min(split * chunk, t_all), t_end = t_lo + min((split + 1) * chunk, t_all);

  const int *table = a.page_table + s * a.table_seq + g * a.table_group;
  const int page_mask = (1 << a.page_shift) - 1;
  const T *Kc = static_cast<const T *>(a.K_cache), *Vc = static_cast<const T *>(a.V_cache);
  const size_t page_step = ((size_t)a.G << a.page_shift) * D, group_off = ((size_t)g << a.page_shift) * D;
  auto entry = [&](int key) { return table[min(key >> a.page_shift, a.max_pages - 1)]; };

  f32x4 acc[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m = kNegInf, l = 0.0f;

  for (int t = t_begin + wv; t < t_end; t += kWaves) {
    const int base = t * kTile;
    int id[2], vid[2];
    bool vok[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      id[h] = entry(base + 16 * h + n);
      id[h] = id[h] >= 0 && id[h] < a.n_pages ? id[h] : -1;
      const int key = base + 16 * h + n;
      O_::row(x.k[h], Kc + max(id[h], 0) * page_step + group_off + (size_t)(key & page_mask) * D, c);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      vid[h] = __shfl(id[h], 4 * c);  // (four keys of a lane group lie in one page: pages hold 8 positions or more)
      vok[h] = vid[h] >= 0;
      const int key = base + 16 * h + 4 * c;
      const T *v = Vc + max(vid[h], 0) * page_step + group_off + (size_t)(key & page_mask) * D;
#pragma unroll
      for (int i = 0; i < 4; ++i) x.load_v(4 * h + i, v + i * D, n);
    }
    const bool whole = __all(vok[0] && vok[1]) && base >= lo && base + kTile - 1 <= hi;
    if (!whole) {  // what lies outside a sequence may hold anything
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = base + 16 * h + 4 * c + i;
          if (!vok[h] || key < lo || key > hi) x.clear_v(4 * h + i);
        }
    }
    float p[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 sc = x.logits(h);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = base + 16 * h + 4 * c + i;
        p[4 * h + i] = vok[h] && key >= my.lo && key <= my.hi ? sc[i] * a.scale2 : kNegInf;
      }
    }
    float mx = p[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, p[i]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float m_new = fmaxf(m, mx);
    const float ref = m_new == kNegInf ? 0.0f : m_new;  // no key seen yet: every exponential is 0
    const float f = __builtin_amdgcn_exp2f(m - ref);
    m = m_new;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(p[i] - ref);
      sum += p[i];
    }
    l = l * f + sum;
#pragma unroll
    for (int j = 0; j < VPT; ++j) acc[j] *= f;
    x.product(p, acc);
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // ---- the four wavefronts' results ----
  if (c == 0) {
    m_s[wv][n] = m;
    l_s[wv][n] = l;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < VPT; ++j)
      if (VPT * (4 * c + i) + j < D) acc_s[wv][n][VPT * (4 * c + i) + j] = acc[j][i];
  __syncthreads();
  for (int e = threadIdx.x; e < kRows * D; e += 64 * kWaves) {
    const int r = e / D, ch = e % D;
    if (row0 + r >= rows) break;
    float mm = m_s[0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, m_s[w][r]);
    const float ref = mm == kNegInf ? 0.0f : mm;
    float ll = 0.0f, o = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(m_s[w][r] - ref);
      ll += l_s[w][r] * f;
      o += acc_s[w][r][ch] * f;
    }
    const int tk = PROMPT ? (row0 + r) / a.R : 0;
    const size_t out = (size_t)(tok0 + tk) * a.H + g * a.R + (row0 + r) - tk * a.R;
    if (a.nsplit == 1) {
      store_out(static_cast<T *>(a.O) + out * D + ch, ll == 0.0f ? 0.0f : o / ll);
      if (ch == 0 && a.lse) a.lse[out] = ll == 0.0f ? kNegInf : (mm + __log2f(ll)) * kLn2;
    } else {
      a.part_o[(out * a.nsplit + split) * D + ch] = o;
      if (ch == 0) {
        a.part_ml[(out * a.nsplit + split) * 2] = mm;
        a.part_ml[(out * a.nsplit + split) * 2 + 1] = ll;
      }
    }
  }
}

// Joins a row's parts: a workgroup a row, whose threads take a part each for the weights, and then, 4 channels each, every
// (256 / (d / 4))-th part's sums.  Parts that met no key have weight 0 and finite sums.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_kernel(Args a, int tokens)
{
  constexpr int LANES = D / 4, GROUPS = 256 / LANES;
  __shared__ float red_s[4], l_s[4], w_s[kMostSplits];
  __shared__ __attribute__((aligned(16))) float4 o_s[GROUPS][LANES];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int row = blockIdx.x;
  if (tokens && row / a.H >= token_at(a, a.S)) return;  // (a row that no sequence owns stays as it is)
  const float *ml = a.part_ml + (size_t)row * a.nsplit * 2;
  const float4 *po = reinterpret_cast<const float4 *>(a.part_o + (size_t)row * a.nsplit * D);
  const bool mine = tid < a.nsplit;
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
  if (mine) w_s[tid] = w;
  if (lane == 0) l_s[wv] = l;
  __syncthreads();
  l = (l_s[0] + l_s[1]) + (l_s[2] + l_s[3]);
  const int at = tid % LANES, grp = tid / LANES;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int i = grp; i < a.nsplit; i += GROUPS) {
    const float4 v = po[(size_t)i * LANES + at];
    const float f = w_s[i];
    o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
  }
  o_s[grp][at] = o;
  __syncthreads();
  if (tid < D) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) sum += reinterpret_cast<const float *>(&o_s[i][0])[tid];
    store_out(static_cast<T *>(a.O) + (size_t)row * D + tid, l == 0.0f ? 0.0f : sum / l);
  }
  if (tid == 0 && a.lse) a.lse[row] = l == 0.0f ? kNegInf : (m + __log2f(l)) * kLn2;
}

int attn_splits(const Args &a, bool prompt)
{
  if (prompt) return 1;
  const long base = (long)a.S * a.G * ((a.R + kRows - 1) / kRows);
  const long tiles = ((long)(a.window < a.cap ? a.window + kTile - 1 : a.cap) + kTile - 1) / kTile;
  const long want = (1024 + base - 1) / base, most = (tiles + 2 * kWaves - 1) / (2 * kWaves);
  const long n = want < most ? want : most;
  return (int)(n < 1 ? 1 : (n > kMostSplits ? kMostSplits : n));
}

namespace {

template <typename T, int D>
void launch_rows(const Args &a, bool prompt, hipStream_t st)
{
  const long tiles = prompt ? (long)a.T * a.R / kRows + a.S : (long)a.S * ((a.R + kRows - 1) / kRows);
  const dim3 grid((unsigned)(tiles * a.nsplit * a.G)), block(64 * kWaves);
  if (prompt) BLOSSOM_LAUNCH((rows_kernel<T, D, true>), grid, block, 0, st, a);
  else BLOSSOM_LAUNCH((rows_kernel<T, D, false>), grid, block, 0, st, a);
  if (a.nsplit > 1) {
    const long rows = (long)(prompt ? a.T : a.S) * a.H;
    BLOSSOM_LAUNCH((join_kernel<T, D>), dim3((unsigned)rows), dim3(256), 0, st, a, prompt ? a.T : 0);
  }
}

template <typename T>
void launch_rows_d(const Args &a, bool prompt, hipStream_t st)
{
  switch (a.d) {
    case 8: launch_rows<T, 8>(a, prompt, st); break;
    case 16: launch_rows<T, 16>(a, prompt, st); break;
    case 32: launch_rows<T, 32>(a, prompt, st); break;
    case 64: launch_rows<T, 64>(a, prompt, st); break;
    default: launch_rows<T, 128>(a, prompt, st); break;
  }
}

}  // namespace

void launch_decode(const Args &a, hipStream_t st)
{
  if (a.dtype == 0) launch_rows_d<float>(a, false, st);
  else launch_rows_d<bf16_t>(a, false, st);
}

void launch_prompt(const Args &a, hipStream_t st)
{
  if (prompt_mfma_supported(a)) return launch_prompt_mfma(a, st);
  if (a.dtype == 0) launch_rows_d<float>(a, true, st);
  else launch_rows_d<bf16_t>(a, true, st);
}

}  // namespace paged
}  // namespace blossom
