// Projection with low-rank adapters of many requests (include/iodf.h: iodf_proj_forward).
#include "proj_kernel.h"

namespace iodf {
namespace {

// sum over 16 products of 8-bit integers
template <bool kUnsigned>
__device__ __forceinline__ int dot4(int w, int x, int acc) {
  if (kUnsigned) asm("dp4a.s32.u32 %0, %1, %2, %3;" : "=r"(acc) : "r"(w), "r"(x), "r"(acc));
  else asm("dp4a.s32.s32 %0, %1, %2, %3;" : "=r"(acc) : "r"(w), "r"(x), "r"(acc));
  return acc;
}

// 16 bytes of a row of x from channel k0 on; channels beyond the last are zero and not read
__device__ __forceinline__ int4 load_x16(const uint8_t* row, int k0, int K) {
  if (k0 + 16 <= K) return *reinterpret_cast<const int4*>(row + k0);
  int w[4] = {0, 0, 0, 0};
  for (int i = 0; k0 + i < K; ++i) w[i >> 2] |= (int)row[k0 + i] << (8 * (i & 3));
  return make_int4(w[0], w[1], w[2], w[3]);
}

template <bool kUnsigned>
__device__ __forceinline__ int dot_row(const int8_t* w, const uint8_t* x, int K, int k0, int step) {
  int acc = 0;
  for (int k = k0; k < K; k += step) {
    const int4 a = *reinterpret_cast<const int4*>(w + k), b = load_x16(x, k, K);
    acc = dot4<kUnsigned>(a.x, b.x, acc);
    acc = dot4<kUnsigned>(a.y, b.y, acc);
    acc = dot4<kUnsigned>(a.z, b.z, acc);
    acc = dot4<kUnsigned>(a.w, b.w, acc);
  }
  return acc;
}

// Which adapter a row uses: the last request that starts at or before it, found by halving. Any content of
// seg_start gives some request 0 <= q < n_seg, so nothing beyond the arrays is read.
__device__ __forceinline__ int slot_of_row(const ProjArgs& a, int row) {
  int lo = 0, hi = a.n_seg - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.seg_start[mid] <= row) lo = mid;
    else hi = mid - 1;
  }
  if (row < a.seg_start[lo] || row >= a.seg_start[lo + 1]) return -2;
  const int s = a.seg_adapter[lo];
  return s >= 0 && s < a.max_adapters && a.rank[s] > 0 ? s : -1;
}

// h of every row, a warp per row; block 0 looks the requests over
template <bool kUnsigned>
__global__ void __launch_bounds__(128) down_kernel(const ProjArgs a) {
  if (blockIdx.x == 0)
    for (int q = threadIdx.x; q < a.n_seg; q += blockDim.x) {
      const int s0 = a.seg_start[q], s1 = a.seg_start[q + 1], ad = a.seg_adapter[q];
      if (s0 < 0 || s1 < s0 || s1 > a.rows || ad < -1 || ad >= a.max_adapters) atomicAdd(a.status + 1, 1u);
    }
  const int lane = threadIdx.x & 31;
  for (int row = blockIdx.x * 4 + (threadIdx.x >> 5); row < a.rows; row += gridDim.x * 4) {
    const int slot = slot_of_row(a, row);
    if (lane == 0) a.row_slot[row] = slot;
    if (slot < 0) continue;
    const int R = a.rank[slot];
    for (int j = 0; j < R; ++j) {
      const size_t i = (size_t)slot * a.max_rank + j;
      int acc = dot_row<kUnsigned>(a.down + i * a.kp, a.x + (size_t)row * a.ldx, a.k, lane * 16, 512);
      for (int o = 16; o; o >>= 1) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, o);
      if (lane == 0) {
        const int2 q = a.down_rq[i];
        const int v = (int)(((long long)acc * q.x + (1ll << (30 + q.y))) >> (31 + q.y));
        a.h[(size_t)row * a.max_rank + j] = (int8_t)min(max(v, -128), 127);
      }
    }
  }
}

template <bool kUnsigned>
__global__ void __launch_bounds__(128) proj_rows_kernel(const ProjArgs a) {
  const long long total = (long long)a.rows * a.n;
  for (long long i = (long long)blockIdx.x * 128 + threadIdx.x; i < total; i += (long long)gridDim.x * 128) {
    const int row = (int)(i / a.n), n = (int)(i % a.n);
    const int slot = a.n_seg ? a.row_slot[row] : -1;
    if (slot == -2) continue;
    int acc = dot_row<kUnsigned>(a.w + (size_t)n * a.kp, a.x + (size_t)row * a.ldx, a.k, 0, 16);
    if (slot >= 0) {
      const int R = a.rank[slot];
      const int8_t* up = a.up + ((size_t)slot * a.n + n) * a.max_rank;
      const int8_t* h = a.h + (size_t)row * a.max_rank;
      for (int j = 0; j < R; ++j) acc += (int)up[j] * h[j];
    }
    const int4 q = a.rq[n];
    const long long add = (long long)(((unsigned long long)(uint32_t)q.w << 32) | (uint32_t)q.z);
    const int v = min(max((int)(((long long)acc * q.x + add) >> (31 + q.y)), a.lo), a.hi);
    const size_t o = (size_t)row * a.ldy + n;
    if (a.y_bytes == 1) ((uint8_t*)a.y)[o] = (uint8_t)v;
    else ((int*)a.y)[o] = v;
  }
}

template <bool kUnsigned>
cudaError_t launch(const ProjArgs& a, cudaStream_t stream) {
  if (a.n_seg) {
    const int grid = (a.rows + 3) / 4 < 148 * 16 ? (a.rows + 3) / 4 : 148 * 16;
    down_kernel<kUnsigned><<<grid, 128, 0, stream>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  const long long blocks = ((long long)a.rows * a.n + 127) / 128;
  proj_rows_kernel<kUnsigned><<<(int)(blocks < 148 * 64 ? blocks : 148 * 64), 128, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_proj(const ProjArgs& a, cudaStream_t stream) {
  return a.x_unsigned ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace iodf
