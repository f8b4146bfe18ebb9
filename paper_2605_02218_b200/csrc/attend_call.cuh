// A call of the attention over the paged cache, as the host part of the library hands it to the kernels of its type; the two types are
// compiled on their own (attend_bf16.cu, attend_f16.cu), side by side.
#pragma once
#include "attend_common.cuh"
#include "covspec.h"

namespace covspec {
namespace attend {

// Largest request, as rows of a key head, that the kernel for few rows takes when both run; its CTAs at most per SM.
constexpr int kFewRows = 64, kRowsCtas = 2;
constexpr int kWideRows = 256, kWideKeys = 128;   // an item's rows and a unit's keys in the kernel for many rows

struct Call {
  Params few, many;              // what each of the two kernels is given
  const covspec_cache* cache;
  int rows;                      // of an item in the kernel for few rows: 16, 32 or 64
  int ctas, many_ctas;           // many_ctas 0: that kernel is not needed
  cudaStream_t stream;
};
cudaError_t launch_bf16(const Call& call);
cudaError_t launch_f16(const Call& call);

}  // namespace attend
}  // namespace covspec
