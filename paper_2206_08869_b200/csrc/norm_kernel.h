// Norms before and after a block with its gate and residual scale: launch arguments.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace iodf {

struct ViewArgs {                     // element (row, c) at img * (row / pixels) + chan * c + pix * (row % pixels)
  long long pixels, img, chan, pix;
};

struct NormArgs {
  const void* r;
  void* r_out;
  ViewArgs rv, ov;
  const void* b;
  const uint8_t* gate;
  void* n;
  long long ldb, ldg, ldn;
  long long rows;
  int channels;
  int res_i16, block_i8, has_block;
  int post, pre;                      // 0, IODF_NORM_RMS, IODF_NORM_CENTRED
  int shift, n_shift;
  int res_lo, res_hi, n_lo, n_hi;
  int n_type;                         // IODF_I8 or IODF_U8
  int n_full;                         // the clip of n is its type's range
  unsigned long long eps;
  const int32_t *mult, *n_mult, *n_bias;   // device, [channels]
};

cudaError_t launch_norm(const NormArgs& a, cudaStream_t stream);

}  // namespace iodf
