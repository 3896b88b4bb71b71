// C ABI of the paged key/value cache's operators: argument checks (before any HIP call), workspace sizes, dispatch.
// See include/blossom.h for the contract.
#include "../../include/blossom.h"

#include <cmath>

#include "paged.h"

using namespace blossom::paged;

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_params(const blossom_paged_params *p, Args *a)
{
  if (!p) return BLOSSOM_ERR_NULL;
  if (p->S < 1 || p->T < 1 || p->H < 1 || p->G < 1 || p->n_pages < 1 || p->max_pages < 1) return BLOSSOM_ERR_SHAPE;
  if (p->d != 8 && p->d != 16 && p->d != 32 && p->d != 64 && p->d != 128) return BLOSSOM_ERR_UNSUPPORTED;
  if (p->page < 8 || p->page > 256 || (p->page & (p->page - 1))) return BLOSSOM_ERR_UNSUPPORTED;
  if (p->dtype != BLOSSOM_F32 && p->dtype != BLOSSOM_BF16) return BLOSSOM_ERR_UNSUPPORTED;
  if (p->H % p->G != 0 || p->window < 0 || p->max_len < 0 || p->table_per_head < 0 || p->table_per_head > 1)
    return BLOSSOM_ERR_PARAM;
  if (!std::isfinite(p->softmax_scale) || p->softmax_scale < 0.0f) return BLOSSOM_ERR_PARAM;
  // positions and rows are counted in 31 bits, with room for a tile more
  const int64_t most = 0x7FFFFFFFll - 4096, held = (int64_t)p->max_pages * p->page;
  if (held > most || (int64_t)p->T * p->H > most || (int64_t)p->S * p->H > most) return BLOSSOM_ERR_SHAPE;
  *a = Args{};
  a->S = p->S; a->T = p->T; a->H = p->H; a->G = p->G; a->R = p->H / p->G; a->d = p->d;
  a->by_G = divisor(a->G); a->by_H = divisor(a->H); a->by_R = divisor(a->R);
  a->page_shift = __builtin_ctz((unsigned)p->page);
  a->n_pages = p->n_pages; a->max_pages = p->max_pages;
  a->cap = p->max_len > 0 && p->max_len < held ? p->max_len : (int)held;
  a->window = p->window > 0 ? p->window : 0x7FFFFFFF;
  a->dtype = p->dtype;
  a->scale2 = (p->softmax_scale > 0.0f ? p->softmax_scale : 1.0f / std::sqrt((float)p->d)) * 1.4426950408889634f;
  a->table_group = p->table_per_head ? p->max_pages : 0;
  a->table_seq = (int64_t)p->max_pages * (p->table_per_head ? p->G : 1);
  return BLOSSOM_OK;
}

// A token stride in elements: 0 means rows one after another.
int check_stride(const Args &a, int64_t given, int heads, int64_t *stride)
{
  const int64_t row = (int64_t)heads * a.d;
  *stride = given == 0 ? row : given;
  if (*stride < row) return BLOSSOM_ERR_PARAM;
  return *stride % (a.dtype == BLOSSOM_F32 ? 4 : 8) == 0 ? BLOSSOM_OK : BLOSSOM_ERR_ALIGN;
}

// partial results: rows of them, and their bytes
size_t part_rows(const Args &a, bool prompt) { return (size_t)a.H * a.parts * (prompt ? a.T : 1); }
size_t attn_ws_bytes(Args &a, bool prompt)
{
  a.parts = prompt ? prompt_parts(a) : decode_parts(a);
  if (a.parts <= (prompt ? 1 : 0)) return 0;
  return part_rows(a, prompt) * (a.d + 2) * sizeof(float) + (prompt ? 0 : (size_t)a.S * sizeof(int2));
}

// trees: partial results, then where each token's are
size_t tree_ws_bytes(const Args &a)
{
  const size_t rows = tree_part_rows(a);
  return rows ? rows * (a.d + 2) * sizeof(float) + (1 + (size_t)a.T) * sizeof(int4) : 0;
}

int launch_status() { return hipGetLastError() == hipSuccess ? BLOSSOM_OK : BLOSSOM_ERR_LAUNCH; }

int attn(const blossom_paged_params *p, bool prompt, const void *Q, int64_t q_stride, const void *K_cache, const void *V_cache,
         const int32_t *page_table, const int32_t *cu_seqlens, const int32_t *kv_len, void *O, float *lse, void *ws,
         size_t ws_bytes, void *hip_stream)
{
  Args a;
  int rc = check_params(p, &a);
  if (rc) return rc;
  if (prompt && p->table_per_head) return BLOSSOM_ERR_UNSUPPORTED;
  if (!Q || !K_cache || !V_cache || !page_table || !kv_len || !O || (prompt && !cu_seqlens)) return BLOSSOM_ERR_NULL;
  if (!aligned16(Q) || !aligned16(K_cache) || !aligned16(V_cache) || !aligned16(O)) return BLOSSOM_ERR_ALIGN;
  rc = check_stride(a, q_stride, a.H, &a.q_stride);
  if (rc) return rc;
  const size_t need = attn_ws_bytes(a, prompt);
  a.by_parts = divisor(a.parts > 0 ? a.parts : 1);
  if (need) {
    if (!ws || ws_bytes < need) return BLOSSOM_ERR_WORKSPACE;
    if (!aligned16(ws)) return BLOSSOM_ERR_ALIGN;
    a.part_o = static_cast<float *>(ws);
    a.part_ml = a.part_o + part_rows(a, prompt) * a.d;
    a.part_of = reinterpret_cast<int2 *>(a.part_ml + part_rows(a, prompt) * 2);
  }
  a.Q = Q; a.K_cache = const_cast<void *>(K_cache); a.V_cache = const_cast<void *>(V_cache);
  a.page_table = page_table; a.cu = cu_seqlens; a.kv_len = kv_len;
  a.O = O; a.lse = lse;
  (void)hipGetLastError();  // an earlier call's error is not this one's
  if (!(prompt ? launch_prompt : launch_decode)(a, (hipStream_t)hip_stream)) return BLOSSOM_ERR_SHAPE;
  return launch_status();
}

int append(const blossom_paged_params *p, const void *Q, int64_t q_stride, const void *K, int64_t k_stride, const void *V, int64_t v_stride,
           const float *rope_cos, const float *rope_sin, const int32_t *page_table, const int32_t *cu_seqlens, const int32_t *kv_len,
           const int64_t *tree_mask, void *K_cache, void *V_cache, void *Q_rot, void *hip_stream)
{
  Args a;
  int rc = check_params(p, &a);
  if (rc) return rc;
  if (p->table_per_head) return BLOSSOM_ERR_UNSUPPORTED;
  if (!K || !V || !page_table || !cu_seqlens || !kv_len || !K_cache || !V_cache) return BLOSSOM_ERR_NULL;
  if (!rope_cos != !rope_sin || !Q != !Q_rot || (Q && !rope_cos)) return BLOSSOM_ERR_NULL;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(rope_cos) || !aligned16(rope_sin) || !aligned16(K_cache) ||
      !aligned16(V_cache) || !aligned16(Q_rot))
    return BLOSSOM_ERR_ALIGN;
  rc = check_stride(a, q_stride, a.H, &a.q_stride);
  if (!rc) rc = check_stride(a, k_stride, a.G, &a.k_stride);
  if (!rc) rc = check_stride(a, v_stride, a.G, &a.v_stride);
  if (rc) return rc;
  a.Q = Q; a.K = K; a.V = V; a.rope_cos = rope_cos; a.rope_sin = rope_sin;
  a.page_table = page_table; a.cu = cu_seqlens; a.kv_len = kv_len; a.tree = tree_mask;
  a.K_cache = K_cache; a.V_cache = V_cache; a.Q_rot = Q_rot;
  (void)hipGetLastError();
  if (!launch_append(a, (hipStream_t)hip_stream)) return BLOSSOM_ERR_SHAPE;
  return launch_status();
}

// the fork's workspace: where a sequence's own pages begin, which of them it asks for and how many, copies that read a page
int fork_chunks(const Args &a) { return (a.max_pages + 63) / 64; }
size_t fork_ws_bytes(const Args &a, int n_new)
{
  return (size_t)n_new * (sizeof(int4) + fork_chunks(a) * sizeof(uint4) + sizeof(int)) + a.n_pages * sizeof(int);
}

bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace

extern "C" {

size_t blossom_paged_workspace_bytes(const blossom_paged_params *p, int which)
{
  Args a;
  if (check_params(p, &a) != BLOSSOM_OK || (which != BLOSSOM_WS_DECODE && which != BLOSSOM_WS_PROMPT && which != BLOSSOM_WS_TREE)) return 0;
  if (which == BLOSSOM_WS_TREE) {
    plan_tree(a);
    return tree_ws_bytes(a);
  }
  return attn_ws_bytes(a, which == BLOSSOM_WS_PROMPT);
}

int blossom_kv_append(const blossom_paged_params *p, const void *Q, int64_t q_stride, const void *K, int64_t k_stride,
                      const void *V, int64_t v_stride, const float *rope_cos, const float *rope_sin,
                      const int32_t *page_table, const int32_t *cu_seqlens, const int32_t *kv_len, void *K_cache,
                      void *V_cache, void *Q_rot, void *hip_stream)
{
  return append(p, Q, q_stride, K, k_stride, V, v_stride, rope_cos, rope_sin, page_table, cu_seqlens, kv_len, nullptr, K_cache, V_cache,
                Q_rot, hip_stream);
}

int blossom_kv_append_tree(const blossom_paged_params *p, const void *Q, int64_t q_stride, const void *K, int64_t k_stride,
                           const void *V, int64_t v_stride, const float *rope_cos, const float *rope_sin,
                           const int32_t *page_table, const int32_t *cu_seqlens, const int32_t *kv_len,
                           const int64_t *tree_mask, void *K_cache, void *V_cache, void *Q_rot, void *hip_stream)
{
  if (!tree_mask) return BLOSSOM_ERR_NULL;
  if (!aligned(tree_mask, 8)) return BLOSSOM_ERR_ALIGN;
  return append(p, Q, q_stride, K, k_stride, V, v_stride, rope_cos, rope_sin, page_table, cu_seqlens, kv_len, tree_mask, K_cache, V_cache,
                Q_rot, hip_stream);
}

int blossom_attn_decode(const blossom_paged_params *p, const void *Q, int64_t q_stride, const void *K_cache,
                        const void *V_cache, const int32_t *page_table, const int32_t *kv_len, void *O, float *lse,
                        void *ws, size_t ws_bytes, void *hip_stream)
{
  return attn(p, false, Q, q_stride, K_cache, V_cache, page_table, nullptr, kv_len, O, lse, ws, ws_bytes, hip_stream);
}

int blossom_attn_prompt(const blossom_paged_params *p, const void *Q, int64_t q_stride, const void *K_cache,
                        const void *V_cache, const int32_t *page_table, const int32_t *cu_seqlens, const int32_t *kv_len,
                        void *O, float *lse, void *ws, size_t ws_bytes, void *hip_stream)
{
  return attn(p, true, Q, q_stride, K_cache, V_cache, page_table, cu_seqlens, kv_len, O, lse, ws, ws_bytes, hip_stream);
}

int blossom_attn_tree(const blossom_paged_params *p, const void *Q, int64_t q_stride, const void *K_cache, const void *V_cache,
                      const int32_t *page_table, const int32_t *cu_seqlens, const int32_t *kv_len, const int64_t *tree_mask,
                      void *O, float *lse, void *ws, size_t ws_bytes, void *hip_stream)
{
  Args a;
  int rc = check_params(p, &a);
  if (rc) return rc;
  if (p->table_per_head) return BLOSSOM_ERR_UNSUPPORTED;
  if (!Q || !K_cache || !V_cache || !page_table || !cu_seqlens || !kv_len || !tree_mask || !O) return BLOSSOM_ERR_NULL;
  if (!aligned16(Q) || !aligned16(K_cache) || !aligned16(V_cache) || !aligned16(O) || !aligned(tree_mask, 8)) return BLOSSOM_ERR_ALIGN;
  rc = check_stride(a, q_stride, a.H, &a.q_stride);
  if (rc) return rc;
  plan_tree(a);
  const size_t need = tree_ws_bytes(a);
  if (need) {
    if (!ws || ws_bytes < need) return BLOSSOM_ERR_WORKSPACE;
    if (!aligned16(ws)) return BLOSSOM_ERR_ALIGN;
    a.part_at = static_cast<int4 *>(ws);
    a.part_o = reinterpret_cast<float *>(a.part_at + 1 + a.T);
    a.part_ml = a.part_o + tree_part_rows(a) * a.d;
  }
  a.Q = Q; a.K_cache = const_cast<void *>(K_cache); a.V_cache = const_cast<void *>(V_cache);
  a.page_table = page_table; a.cu = cu_seqlens; a.kv_len = kv_len; a.tree = tree_mask;
  a.O = O; a.lse = lse;
  (void)hipGetLastError();
  if (!launch_tree(a, (hipStream_t)hip_stream)) return BLOSSOM_ERR_SHAPE;
  return launch_status();
}

int blossom_kv_accept(const blossom_paged_params *p, int32_t keep_width, const int32_t *keep, const int32_t *page_table,
                      const int32_t *cu_seqlens, const int32_t *kv_len, void *K_cache, void *V_cache, int32_t *new_len,
                      void *hip_stream)
{
  Args a;
  const int rc = check_params(p, &a);
  if (rc) return rc;
  if (p->table_per_head) return BLOSSOM_ERR_UNSUPPORTED;
  if (keep_width < 1) return BLOSSOM_ERR_SHAPE;
  if (!keep || !page_table || !cu_seqlens || !kv_len || !K_cache || !V_cache) return BLOSSOM_ERR_NULL;
  if (new_len == kv_len) return BLOSSOM_ERR_PARAM;
  if (!aligned16(K_cache) || !aligned16(V_cache)) return BLOSSOM_ERR_ALIGN;
  a.page_table = page_table; a.cu = cu_seqlens; a.kv_len = kv_len;
  a.K_cache = K_cache; a.V_cache = V_cache;
  (void)hipGetLastError();
  if (!launch_accept(a, Accept{keep, keep_width, new_len}, (hipStream_t)hip_stream)) return BLOSSOM_ERR_SHAPE;
  return launch_status();
}

size_t blossom_fork_workspace_bytes(const blossom_paged_params *p, int32_t n_new)
{
  Args a;
  return check_params(p, &a) == BLOSSOM_OK && n_new >= 1 ? fork_ws_bytes(a, n_new) : 0;
}

int blossom_kv_fork(const blossom_paged_params *p, int32_t n_new, int32_t grow, const int32_t *parent, const int32_t *page_table,
                    const int32_t *kv_len, const int32_t *refs, int32_t *new_table, int32_t *new_len, int32_t *new_refs,
                    int32_t *copies, int32_t *missing, void *ws, size_t ws_bytes, void *hip_stream)
{
  Args a;
  const int rc = check_params(p, &a);
  if (rc) return rc;
  if (p->table_per_head) return BLOSSOM_ERR_UNSUPPORTED;
  if (n_new < 1 || (int64_t)n_new * a.max_pages > 0x7FFFFFFFll || (int64_t)a.S * a.max_pages > 0x7FFFFFFFll) return BLOSSOM_ERR_SHAPE;
  if (grow < 0) return BLOSSOM_ERR_PARAM;
  if (!parent || !page_table || !kv_len || !refs || !new_table || !new_len || !new_refs || !copies || !missing) return BLOSSOM_ERR_NULL;
  if (new_table == page_table || new_len == kv_len || new_refs == refs) return BLOSSOM_ERR_PARAM;
  if (!ws || ws_bytes < fork_ws_bytes(a, n_new)) return BLOSSOM_ERR_WORKSPACE;
  if (!aligned16(ws)) return BLOSSOM_ERR_ALIGN;
  a.page_table = page_table; a.kv_len = kv_len;
  Fork x{};
  x.N = n_new; x.grow = grow; x.parent = parent; x.refs = refs;
  x.table = new_table; x.len = new_len; x.new_refs = new_refs; x.copies = copies; x.missing = missing;
  x.at = static_cast<int4 *>(ws);
  x.asks = reinterpret_cast<uint4 *>(x.at + n_new);
  x.chunks = fork_chunks(a);
  x.fresh = reinterpret_cast<int *>(x.asks + (size_t)n_new * x.chunks);
  x.held = x.fresh + n_new;
  (void)hipGetLastError();
  if (!launch_fork(a, x, (hipStream_t)hip_stream)) return BLOSSOM_ERR_SHAPE;
  return launch_status();
}

int blossom_kv_copy_pages(const blossom_paged_params *p, int32_t n_copies, const int32_t *copies, void *K_cache, void *V_cache,
                          void *hip_stream)
{
  Args a;
  const int rc = check_params(p, &a);
  if (rc) return rc;
  if (n_copies < 1) return BLOSSOM_ERR_SHAPE;
  if (!copies || !K_cache || !V_cache) return BLOSSOM_ERR_NULL;
  if (!aligned16(K_cache) || !aligned16(V_cache)) return BLOSSOM_ERR_ALIGN;
  a.K_cache = K_cache; a.V_cache = V_cache;
  (void)hipGetLastError();
  if (!launch_copy(a, copies, n_copies, (hipStream_t)hip_stream)) return BLOSSOM_ERR_SHAPE;
  return launch_status();
}

}  // extern "C"
