// Projection with low-rank adapters of many requests: launch arguments and the layout of its operands.
//
// Every 8-bit operand of a tcgen05.mma that is a weight is stored as the MMA reads it from shared memory (K-major, no
// swizzle): core matrices of 8 rows x 16 bytes, 128 bytes each; [row / 8][chunk of 16 bytes][8 rows][16]. Consecutive chunks
// are 128 bytes apart (leading-dimension offset), consecutive groups of 8 rows chunks * 128 (stride-dimension offset).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace iodf {

constexpr int kProjTileN = 128;          // output channels per tile: the M of the MMA
constexpr int kProjStage = 128;          // channels (bytes of K) per stage of the ring
constexpr int kProjDownRows = 128;       // rows per tile of the kernel that computes h

struct ProjArgs {
  const uint8_t* x;
  long long ldx, ldy;
  void* y;
  const int32_t *seg_start, *seg_adapter;
  int n_seg, rows;
  int k, n;                            // channels in, out
  int stages, tiles_n;                 // ceil(k / 128), ceil(n / 128)
  int x_unsigned, y_type, y_bytes;     // y_type: IODF_I8, IODF_U8 or IODF_I32
  int lo, hi;                          // ReLU and clip of the layer
  int any_shift;                       // some s is 0
  int max_adapters, max_rank;
  int rp;                              // ranks padded: 32, 64 or 128
  const uint8_t* w;                    // [tiles_n][stages][128 x 128 as above]
  const int4* rq;                      // [tiles_n * 128] {M0, s, addend low, addend high}: y = (acc M0 + addend) >> (31 + s)
  const uint8_t* down;                 // [max_adapters][stages][rp x 128 as above]
  const int2* down_rq;                 // [max_adapters][rp] {M, s}
  const uint8_t* up;                   // [max_adapters][tiles_n][128 x rp as above]
  const int* rank;                     // [max_adapters]
  int8_t* h;                           // workspace [max_rows][rp]
  int* row_slot;                       // workspace [max_rows]: adapter slot (and rank, see kSlotBits), -1 none, -2 in no request
  uint32_t* status;                    // [0] a bounded wait gave up, [1] bad requests
  int sms;
  int clusters[4];                     // clusters of 1, 2, 4, 8 CTAs of the kernel for few rows that run at once
};

// Where element (row, k) of an operand of `width` bytes per row lies.
inline size_t core_offset(size_t row, size_t k, size_t width) {
  return (row / 8) * (width / 16) * 128 + (k / 16) * 128 + (row % 8) * 16 + k % 16;
}

// On the current device, before the first launch; fills sms and clusters.
cudaError_t configure_proj_kernels(int device, ProjArgs* a);

// x_map, x_map_down: CUtensorMaps of x [rows][k] with boxes of 128 bytes x proj_x_rows(a) or kProjDownRows rows and
// the 128-byte swizzle. w_map: of the weights as rows of 128 bytes, box 128 x 128, no swizzle.
int proj_x_rows(const ProjArgs& a);
bool proj_down_tiles(const ProjArgs& a);      // x_map_down is used
cudaError_t launch_proj(const ProjArgs& a, const void* x_map, const void* x_map_down, const void* w_map, cudaStream_t stream);

}  // namespace iodf
