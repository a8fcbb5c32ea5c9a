// Projection with low-rank adapters of many requests: launch arguments.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace iodf {

struct ProjArgs {
  const uint8_t* x;
  long long ldx, ldy;
  void* y;
  const int32_t *seg_start, *seg_adapter;
  int n_seg, rows;
  int k, n, kp;                        // channels in, out; k rounded up to 16
  int x_unsigned, y_bytes;
  int lo, hi;                          // ReLU and clip of the layer
  int max_adapters, max_rank;
  const int8_t* w;                     // [n][kp]
  const int4* rq;                      // [n] {M0, s, addend low, addend high}: y = (acc M0 + addend) >> (31 + s)
  const int8_t* down;                  // [max_adapters][max_rank][kp]
  const int2* down_rq;                 // [max_adapters][max_rank] {M, s}
  const int8_t* up;                    // [max_adapters][n][max_rank]
  const int* rank;                     // [max_adapters]
  int8_t* h;                           // workspace [max_rows][max_rank]
  int* row_slot;                       // workspace [max_rows]: adapter slot, -1 none, -2 in no request
  uint32_t* status;                    // [0] a bounded wait gave up, [1] bad requests
};

cudaError_t launch_proj(const ProjArgs& a, cudaStream_t stream);

}  // namespace iodf
