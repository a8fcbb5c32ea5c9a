// Norms before and after a block with its gate and residual scale (include/iodf.h: iodf_norm_forward).
#include "norm_kernel.h"
#include "../../include/iodf.h"

namespace iodf {
namespace {

constexpr int kLim24 = (1 << 23) - 1;

__device__ __forceinline__ int clip24(int v) { return min(max(v, -kLim24 - 1), kLim24); }

// The two integers that scale a row: N(v) = (v rho + 2^(sh-1)) >> sh with rho / 2^sh ~ 2^22 / sqrt(D), 1 <= D < 2^62.
// sigma = floor(sqrt(D 2^t)) from the root in double precision (off by less than one), put right in integers.
__device__ __forceinline__ void row_scale(unsigned long long D, int* rho, int* sh) {
  const int t = (__clzll((long long)D) - 2) & ~1;
  const unsigned long long m = D << t;
  unsigned long long s = (unsigned long long)sqrt((double)m);
  if (s * s > m) --s;
  if ((s + 1) * (s + 1) <= m) ++s;
  *rho = (int)(((1ull << 61) - 1) / s);
  *sh = 39 - (t >> 1);
}

__device__ __forceinline__ long long block_sum(long long v, long long* red) {
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  long long s = 0;
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) s += red[w];
  return s;
}

// N over the row held in v[0 .. C), in place
__device__ void norm_row(int* v, int C, int kind, unsigned long long eps, long long* red) {
  if (kind == IODF_NORM_CENTRED) {
    long long s = 0;
    for (int c = threadIdx.x; c < C; c += blockDim.x) s += v[c];
    s = 2 * block_sum(s, red) + C;
    long long mean = s / (2 * C);
    if (mean * (2 * C) > s) --mean;
    for (int c = threadIdx.x; c < C; c += blockDim.x) v[c] -= (int)mean;
  }
  long long q = 0;
  for (int c = threadIdx.x; c < C; c += blockDim.x) q += (long long)v[c] * v[c];
  int rho, sh;
  row_scale((unsigned long long)block_sum(q, red) + eps, &rho, &sh);
  for (int c = threadIdx.x; c < C; c += blockDim.x) v[c] = (int)(((long long)v[c] * rho + (1ll << (sh - 1))) >> sh);
}

__device__ __forceinline__ int scaled(int a, int m, int s) {
  return (int)(((long long)a * m + (1ll << (30 + s))) >> (31 + s));
}

__global__ void __launch_bounds__(256) norm_rows_kernel(const NormArgs a) {
  extern __shared__ int v[];
  __shared__ long long red[8];
  const int C = a.channels;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const long long ro = row / a.rv.pixels * a.rv.img + row % a.rv.pixels * a.rv.pix;
    if (a.has_block) {
      for (int c = threadIdx.x; c < C; c += blockDim.x)
        v[c] = a.block_i8 ? ((const int8_t*)a.b)[row * a.ldb + c] : clip24(((const int*)a.b)[row * a.ldb + c]);
      if (a.post) norm_row(v, C, a.post, a.eps, red);
    }
    const long long oo = a.has_block ? row / a.ov.pixels * a.ov.img + row % a.ov.pixels * a.ov.pix : 0;
    for (int c = threadIdx.x; c < C; c += blockDim.x) {
      const long long i = ro + c * a.rv.chan;
      int r = a.res_i16 ? ((const int16_t*)a.r)[i] : clip24(((const int*)a.r)[i]);
      if (a.has_block) {
        const int g = a.gate ? a.gate[row * a.ldg + c] : 1;
        r = min(max(r + scaled(v[c] * g, a.mult[c], a.shift), a.res_lo), a.res_hi);
        const long long o = oo + c * a.ov.chan;
        if (a.res_i16) ((int16_t*)a.r_out)[o] = (int16_t)r;
        else ((int*)a.r_out)[o] = r;
      }
      v[c] = r;
    }
    if (a.pre) {
      norm_row(v, C, a.pre, a.eps, red);
      for (int c = threadIdx.x; c < C; c += blockDim.x)
        ((uint8_t*)a.n)[row * a.ldn + c] = (uint8_t)min(max(scaled(v[c], a.n_mult[c], a.n_shift) + a.n_bias[c], a.n_lo), a.n_hi);
    }
    __syncthreads();
  }
}

}  // namespace

cudaError_t launch_norm(const NormArgs& a, cudaStream_t stream) {
  const int grid = (int)(a.rows < 148 * 64 ? a.rows : 148 * 64);
  norm_rows_kernel<<<grid, 256, sizeof(int) * a.channels, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace iodf
