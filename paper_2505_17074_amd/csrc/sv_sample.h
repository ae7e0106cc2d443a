// Internal declarations of sampling.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sv {

constexpr int kSampleBins = 2048;      // ranges of a histogram
constexpr int kSampleList = 2048;      // tokens of a list
constexpr int kSampleSlabs = 1024;     // runs of ids of a row, at most
constexpr int kSampleSlices = 8;       // slices of a row, at most
constexpr int kSampleShort = 2048;     // 16-byte units of a row that is not cut
constexpr int kSampleWhole = 8192;     // and of one with a top-k in a batch of up to
constexpr int kSampleAlone = 4;        // rows
constexpr int kSampleFirst = 1024;     // a top-k whose tokens are listed whole
constexpr int64_t kSampleHead = 512;   // bytes of a row's workspace before its arrays

// A row's part of the workspace: kSampleHead bytes, then slab, list, hist.
struct SampleRow {
  float* top;                          // [slices] largest values
  int32_t* n;                          // [slices] tokens listed (more than kSampleList: not all of them)
  double* sum;                         // [slices] counts or weights
  char* state;
  char* done;
  double* slab;                        // [kSampleSlabs] weights that stay, by runs of ids
  unsigned long long* list;            // [slices][kSampleList] order and id
  unsigned long long* hist;            // [slices][kSampleBins]
  unsigned long long* group;           // [slices][kSampleBins / 32]
};
inline int64_t sample_row_bytes(int slices) {
  if (slices == 1) return 0;           // it all stays in LDS
  return kSampleHead + 8 * (kSampleSlabs + (int64_t)slices * (kSampleList + kSampleBins + kSampleBins / 32));
}

struct SampleParams {
  const void* logits;
  int64_t stride;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniforms;
  int32_t* tokens;
  void* rows;
  int64_t rows_stride;
  char* work;
  int64_t row_bytes;
  int32_t V;
  int32_t kind;                        // spec_sample_rows_t
  int32_t slices, slice_units;         // 16-byte units of a slice, whole runs of ids
  int32_t slab_units;                  // of a run, a multiple of 64
  int32_t fix;                         // a slice's weights in units of 2^-fix: their sum is below 2^62
};

hipError_t launch_sample(const SampleParams& p, int num_rows, bool f32, hipStream_t s);

}  // namespace sv
