// C ABI of sampling (specsample.h): argument checks and the launch.  Every
// check runs before the first HIP call.
#include "../../include/specsample.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "sv_sample.h"

namespace {

constexpr size_t kAlign = 256;

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
  if (a->num_rows >= 1 << 22) return SPEC_ERR_UNSUPPORTED;                 // a launch's work-items are 32 bits
  return SPEC_OK;
}

// How a row is cut: the fewest runs of ids of 64 units that a list of runs
// holds, and as many slices as give the chip's compute units a work-group each,
// none of less than 1024 units.  One launch in place of three or four is worth
// more where a row is short, and where a few have a top-k, whose rows need no
// sums of weights (fp32, one row of 32000: top-k 50 17 us whole and 22 in eight
// slices; 64 rows, some with top-p alone, 50 whole and 39 in four).
struct SamplePlan {
  int32_t slices, slice_units, slab_units, fix;
  int64_t row_bytes;
  size_t bytes;
};
SamplePlan plan_sample(const spec_sample_args_t* a) {
  SamplePlan P;
  const int64_t vec = a->dtype == SPEC_F32 ? 4 : 8;
  const int64_t units = a->vocab / vec + 2;                 // wherever the row begins
  const int64_t rounds = (units + 64 * sv::kSampleSlabs - 1) / (64 * sv::kSampleSlabs);
  P.slab_units = (int32_t)(64 * rounds);
  const int64_t slabs = (units + P.slab_units - 1) / P.slab_units;
  int64_t slices = std::min<int64_t>(sv::kSampleSlices, 256 / a->num_rows);
  slices = std::max<int64_t>(1, std::min(slices, units / 1024));
  if (units <= sv::kSampleShort || (units <= sv::kSampleWhole && a->top_k && a->num_rows <= sv::kSampleAlone)) slices = 1;
  const int64_t per = (slabs + slices - 1) / slices;
  P.slices = (int32_t)((slabs + per - 1) / per);
  P.slice_units = (int32_t)(per * P.slab_units);
  // a slice of n tokens: weights rounded at 2^-fix, their sum below 2^62
  P.fix = 50;
  while (((int64_t)P.slice_units * vec) >> (62 - P.fix)) --P.fix;
  P.row_bytes = sv::sample_row_bytes(P.slices);
  P.bytes = std::max(kAlign, (size_t)(P.row_bytes * a->num_rows + kAlign - 1) / kAlign * kAlign);
  return P;
}

}  // namespace

extern "C" {

spec_status_t spec_sample_workspace_bytes(const spec_sample_args_t* args, size_t* device_bytes) {
  if (!device_bytes) return SPEC_ERR_INVALID_ARG;
  const spec_status_t st = check_sample(args);
  if (st == SPEC_OK) *device_bytes = plan_sample(args).bytes;
  return st;
}

spec_status_t spec_sample(const spec_sample_args_t* args, void* workspace, size_t workspace_bytes, void* stream) {
  const spec_status_t st = check_sample(args);
  if (st != SPEC_OK) return st;
  const SamplePlan P = plan_sample(args);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % kAlign || workspace_bytes < P.bytes) return SPEC_ERR_WORKSPACE;
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
  p.work = static_cast<char*>(workspace);
  p.row_bytes = P.row_bytes;
  p.slices = P.slices;
  p.slice_units = P.slice_units;
  p.slab_units = P.slab_units;
  p.fix = P.fix;
  return sv::launch_sample(p, args->num_rows, args->dtype == SPEC_F32, static_cast<hipStream_t>(stream)) == hipSuccess
             ? SPEC_OK
             : SPEC_ERR_HIP;
}

}  // extern "C"
