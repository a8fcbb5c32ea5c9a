// Attention over the cache of blocks (include/iodf.h: iodf_attn_forward).
#include "attn.h"

#include <algorithm>

#include "../../include/iodf.h"
#include "attn_device.cuh"
#include "attn_kernels.h"

namespace iodf {

namespace {

// A CTA per row and head, a thread per key and then per dimension.
__global__ void __launch_bounds__(128) row_kernel(const AttnArgs a, const CacheArgs c, const ForwardArgs f) {
  const int row = blockIdx.x, head = blockIdx.y, h = head / a.group, D = a.dim, tid = threadIdx.x;
  __shared__ int p_sh[128], red[8], table_word[kWeightSegments];
  __shared__ long long redl[4];
  __shared__ __align__(16) int8_t q_sh[128];
  if (tid < kWeightSegments) table_word[tid] = weight_word(tid);
  int lo = 0, hi = f.n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (f.row_start[mid + 1] > row) hi = mid;
    else lo = mid + 1;
  }
  if (lo >= f.n || row < f.row_start[lo] || row >= f.row_start[lo + 1]) return;
  const int held = min(max(f.held[lo], 0), f.width * kAttnBlock);
  const int position = held - (f.row_start[lo + 1] - row);
  const Range see = visible(a, position, held);
  if (tid == 0 && f.held[lo] != held) atomicAdd(a.status + 1, 1u);
  if (tid < D) q_sh[tid] = f.q8[((long long)row * a.heads + head) * D + tid];
  const int eq = min((int)f.q_exp[(long long)row * a.heads + head], kAttnMaxExp);
  __syncthreads();
  const int b0 = see.first / kAttnBlock, b1 = see.last <= see.first ? b0 : (see.last + kAttnBlock - 1) / kAttnBlock;
  int T = INT32_MIN, V = 0;
  long long A = 0, L = 0;
  for (int pass = 0; pass < 2; ++pass) {
    for (int b = b0; b < b1; ++b) {
      const int id = f.table[(long long)lo * f.ldt + b];
      if ((unsigned)id >= (unsigned)c.blocks) {
        if (pass && tid == 0) atomicAdd(a.status + 1, 1u);
        continue;
      }
      const long long at = (long long)id * a.kv + h;
      const int ek = min((int)c.k_exp[at], kAttnMaxExp), ev = min((int)c.v_exp[at], kAttnMaxExp);
      const int key = b * kAttnBlock + tid;
      const bool seen = key >= see.first && key < see.last;
      int s = 0;
      const int4* k = reinterpret_cast<const int4*>(c.k + (at * kAttnBlock + tid) * D);
      for (int i = 0; i < D / 16; ++i) {
        const int4 kv = k[i], qv = reinterpret_cast<const int4*>(q_sh)[i];
        s = __dp4a(kv.x, qv.x, s); s = __dp4a(kv.y, qv.y, s); s = __dp4a(kv.z, qv.z, s); s = __dp4a(kv.w, qv.w, s);
      }
      const int t = score_octaves(s, score_multiplier(a.score_m0, eq + ek, a.score_s));
      if (pass == 0) {
        if (seen) T = max(T, t);
        V = max(V, ev);
      } else {
        int n = seen ? max(t - T - 8192 * (V - ev), kWeightLow) : kWeightLow;
        const int p = (int)(weight_bits(n, table_word[(n >> 7) & 63]) - kWeightBias);
        p_sh[tid] = p;
        L += (long long)p << (V - ev);
        __syncthreads();
        if (tid < D) {
          const int8_t* v = c.v + (at * D + tid) * kAttnBlock;
          for (int j = 0; j < kAttnBlock; ++j) A += (long long)p_sh[j] * v[j];
        }
        __syncthreads();
      }
    }
    if (pass == 0) {
      T = __reduce_max_sync(0xFFFFFFFFu, T);
      if (tid % 32 == 0) red[tid / 32] = T;
      __syncthreads();
      T = max(max(red[0], red[1]), max(red[2], red[3]));
    }
  }
  for (int d = 16; d; d /= 2) L += __shfl_xor_sync(0xFFFFFFFFu, L, d);
  if (tid % 32 == 0) redl[tid / 32] = L;
  __syncthreads();
  L = redl[0] + redl[1] + redl[2] + redl[3];
  if (tid >= D) return;
  const int o = L ? quotient(A, reciprocal(L, V)) : 0;
  const int y = requantised(o, a.out[head * D + tid], a.lo, a.hi);
  const long long at = (long long)row * f.ldy + head * D + tid;
  if (a.y_bytes == 1) ((int8_t*)f.y)[at] = (int8_t)y;
  else ((int*)f.y)[at] = y;
}

}  // namespace

cudaError_t configure_attn_kernels(int device, AttnArgs* a) {
  cudaError_t e = cudaDeviceGetAttribute(&a->sms, cudaDevAttrMultiProcessorCount, device);
  if (e == cudaSuccess) e = configure_attn_cache();
  return e == cudaSuccess ? configure_attn_tile() : e;
}

cudaError_t launch_attn_forward(const AttnArgs& a, const CacheArgs& c, const ForwardArgs& f, const CUtensorMap& k_map, const CUtensorMap& v_map,
                                cudaStream_t stream) {
  if ((long long)f.rows * a.group >= 0ll * f.n) return launch_attn_tile(a, c, f, k_map, v_map, stream);
  row_kernel<<<dim3((unsigned)f.rows, (unsigned)a.heads), 128, 0, stream>>>(a, c, f);
  return cudaGetLastError();
}

}  // namespace iodf
