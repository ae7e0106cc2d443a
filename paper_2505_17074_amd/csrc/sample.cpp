// C ABI of sampling (specsample.h): argument checks and the launch.  Every
// check runs before the first HIP call.
#include "../../include/specsample.h"

#include <hip/hip_runtime.h>

#include "sv_sample.h"

namespace {

spec_status_t check_sample(const spec_sample_args_t* a) {
  if (!a || a->num_rows < 1 || a->vocab < 1) return SPEC_ERR_INVALID_ARG;
  if (a->dtype != SPEC_F32 && a->dtype != SPEC_BF16) return SPEC_ERR_INVALID_ARG;
  if (a->rows_kind != SPEC_SAMPLE_NONE && a->rows_kind != SPEC_SAMPLE_PROBS && a->rows_kind != SPEC_SAMPLE_LOGITS)
    return SPEC_ERR_INVALID_ARG;
  const uintptr_t eb = a->dtype == SPEC_F32 ? 4 : 2;
  auto is = [](const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; };
  if (!a->logits || !is(a->logits, eb)) return SPEC_ERR_INVALID_ARG;
  if (a->num_rows > 1 && a->logits_stride < a->vocab) return SPEC_ERR_INVALID_ARG;
  if (!is(a->temperature, 4) || !is(a->top_k, 4) || !is(a->top_p, 4) || !is(a->min_p, 4) || !is(a->uniforms, 4) ||
      !is(a->tokens, 4))
    return SPEC_ERR_INVALID_ARG;
  if (a->tokens && !a->uniforms) return SPEC_ERR_INVALID_ARG;
  if (a->rows_kind != SPEC_SAMPLE_NONE) {
    if (!a->rows || !is(a->rows, eb)) return SPEC_ERR_INVALID_ARG;
    if (a->num_rows > 1 && a->rows_stride < a->vocab) return SPEC_ERR_INVALID_ARG;
    if (a->rows == a->logits && a->num_rows > 1 && a->rows_stride != a->logits_stride) return SPEC_ERR_INVALID_ARG;
  } else if (!a->tokens) {
    return SPEC_ERR_INVALID_ARG;           // nothing to do
  }
  // a row's ids and places are 32 bits, a sum of its weights 62
  if (a->vocab > 1 << 28) return SPEC_ERR_UNSUPPORTED;
  return SPEC_OK;
}

}  // namespace

extern "C" {

spec_status_t spec_sample_workspace_bytes(const spec_sample_args_t* args, size_t* device_bytes) {
  if (!device_bytes) return SPEC_ERR_INVALID_ARG;
  const spec_status_t st = check_sample(args);
  if (st == SPEC_OK) *device_bytes = 0;
  return st;
}

spec_status_t spec_sample(const spec_sample_args_t* args, void* workspace, size_t workspace_bytes, void* stream) {
  const spec_status_t st = check_sample(args);
  if (st != SPEC_OK) return st;
  (void)workspace;
  (void)workspace_bytes;
  sv::SampleParams p{};
  p.logits = args->logits;
  p.stride = args->logits_stride;
  p.temperature = args->temperature;
  p.top_k = args->top_k;
  p.top_p = args->top_p;
  p.min_p = args->min_p;
  p.uniforms = args->uniforms;
  p.tokens = args->tokens;
  p.rows = args->rows;
  p.rows_stride = args->rows_stride;
  p.V = args->vocab;
  p.kind = args->rows_kind;
  return sv::launch_sample(p, args->num_rows, args->dtype == SPEC_F32, static_cast<hipStream_t>(stream)) == hipSuccess
             ? SPEC_OK
             : SPEC_ERR_HIP;
}

}  // extern "C"
