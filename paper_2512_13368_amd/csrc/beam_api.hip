// C ABI of beam search's selection: argument checks (before any HIP call), workspace size.  See include/blossom.h for the contract.
#include "../../include/blossom.h"

#include "beam.h"

using namespace blossom::beam;

namespace {

int check_params(const blossom_beam_params *p, Args *a)
{
  if (!p) return BLOSSOM_ERR_NULL;
  if (p->B < 1 || p->W < 1 || p->K < 1 || p->V < 1) return BLOSSOM_ERR_SHAPE;
  if (p->W > kMost || p->K > kMost || (p->dtype != BLOSSOM_F32 && p->dtype != BLOSSOM_BF16)) return BLOSSOM_ERR_UNSUPPORTED;
  if ((int64_t)p->B * kMost > 0x7FFFFFFFll) return BLOSSOM_ERR_SHAPE;
  if (p->eos < -1 || p->eos >= p->V) return BLOSSOM_ERR_PARAM;
  *a = Args{};
  a->B = p->B; a->W = p->W; a->K = p->K; a->V = p->V; a->dtype = p->dtype; a->eos = p->eos;
  plan(*a);
  return BLOSSOM_OK;
}

size_t runs(const Args &a) { return (size_t)a.B * a.W * a.lists; }
// (16 where few logits need none: one rule for all callers)
size_t ws_bytes_of(const Args &a) { return a.lists == 0 ? 16 : runs(a) * (sizeof(double2) + a.K * sizeof(unsigned long long)); }
bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace

extern "C" {

size_t blossom_beam_workspace_bytes(const blossom_beam_params *p)
{
  Args a;
  return check_params(p, &a) == BLOSSOM_OK ? ws_bytes_of(a) : 0;
}

int blossom_beam_select(const blossom_beam_params *p, const void *logits, int64_t logits_stride, const float *score, const uint8_t *ended,
                        int32_t *parent, int32_t *token, float *out_score, uint8_t *out_ended, void *ws, size_t ws_bytes, void *hip_stream)
{
  Args a;
  const int rc = check_params(p, &a);
  if (rc) return rc;
  if (!logits || !score || !parent || !token || !out_score) return BLOSSOM_ERR_NULL;
  a.stride = logits_stride == 0 ? a.V : logits_stride;
  if (a.stride < a.V || (ended && a.eos < 0)) return BLOSSOM_ERR_PARAM;
  if (!aligned(logits, a.dtype == BLOSSOM_F32 ? 4 : 2) || !aligned(score, 4) || !aligned(parent, 4) || !aligned(token, 4) || !aligned(out_score, 4))
    return BLOSSOM_ERR_ALIGN;
  if (!ws || ws_bytes < ws_bytes_of(a)) return BLOSSOM_ERR_WORKSPACE;
  if (!aligned(ws, 16)) return BLOSSOM_ERR_ALIGN;
  a.logits = logits; a.score = score; a.ended = ended;
  a.parent = parent; a.token = token; a.out_score = out_score; a.out_ended = out_ended;
  a.stats = static_cast<double2 *>(ws);
  a.lists_of = reinterpret_cast<unsigned long long *>(a.stats + runs(a));
  (void)hipGetLastError();
  if (!launch(a, (hipStream_t)hip_stream)) return BLOSSOM_ERR_SHAPE;
  return hipGetLastError() == hipSuccess ? BLOSSOM_OK : BLOSSOM_ERR_LAUNCH;
}

}  // extern "C"
