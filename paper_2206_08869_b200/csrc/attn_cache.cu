// Before the attention (include/iodf.h: iodf_attn_plan, iodf_attn_append): blocks of the cache for the new tokens of every
// request, and the tokens' keys and values in 8 bits in their places.
#include "attn.h"

#include <algorithm>

#include "../../include/iodf.h"

namespace iodf {
namespace {

// ---- plan ------------------------------------------------------------------------------------------------------
// Prefix sums over the requests, computed by every CTA for itself (16384 requests are 128 KB of input, mostly in L2): of new rows,
// and of blocks taken and given back. Then each CTA fills in its part of the rows and of the table. One launch, no CTA waits for another.
constexpr int kPlanThreads = 512;
constexpr int kPlanRows = 2048;          // of a CTA, about

// Inclusive prefix sum over the CTA's threads; *total over all of them.
__device__ __forceinline__ unsigned long long scanned(unsigned long long v, unsigned long long* warps, unsigned long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const unsigned long long o = __shfl_up_sync(0xFFFFFFFFu, v, d);
    if (lane >= d) v += o;
  }
  __syncthreads();
  if (lane == 31) warps[warp] = v;
  __syncthreads();
  unsigned long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    if (w < warp) before += warps[w];
    all += warps[w];
  }
  *total = all;
  return before + v;
}

__device__ __forceinline__ int blocks_of(int tokens) { return (int)(((long long)tokens + kAttnBlock - 1) / kAttnBlock); }

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanArgs p) {
  extern __shared__ int ends[];                    // [n] end of the request's rows; [n] its first place in the ring, -1: gets nothing
  int* const base = ends + p.n;
  __shared__ unsigned long long warps[kPlanThreads / 32];
  const int tid = threadIdx.x, N = p.ring_size;
  const bool first = blockIdx.x == 0;
  const int head = (int)((unsigned)p.state[0] % (unsigned)N), count = min(max(p.state[1], 0), N);
  unsigned long long rows_before = 0, blocks_before = 0;
  int taken = 0, refused = 0;
  for (int q0 = 0; q0 < p.n; q0 += kPlanThreads) {
    const int q = q0 + tid;
    const int held = q < p.n ? p.held[q] : 0, add = q < p.n ? p.add[q] : 0;
    const bool sane = held >= 0 && held <= p.width * kAttnBlock && add >= -1;
    const int grow = max(add, 0), have = sane ? blocks_of(held) : 0;
    unsigned long long all;
    const unsigned long long end = rows_before + scanned((unsigned long long)grow, warps, &all);
    rows_before += all;
    const long long want = ((long long)held + grow + kAttnBlock - 1) / kAttnBlock;
    const bool ends_now = sane && add == -1;
    const bool fits = sane && add >= 0 && want <= p.width && end <= (unsigned long long)p.rows;
    const int need = fits ? (int)want - have : 0, back = ends_now ? have : 0;
    const unsigned long long sums = blocks_before + scanned((unsigned long long)need | (unsigned long long)back << 32, warps, &all);
    blocks_before += all;
    const int upto = (int)(uint32_t)sums;
    const bool granted = fits && (need == 0 || upto <= count);
    if (q < p.n) {
      ends[q] = (int)min(end, (unsigned long long)p.rows);
      base[q] = granted ? upto - need : -1;
      if (first) {
        p.row_start[q + 1] = ends[q];
        p.held_out[q] = ends_now ? 0 : granted ? held + grow : held;
        refused += !granted && !ends_now;
      }
      if (granted && need) taken = max(taken, upto);
    }
    // Table entries, a request at a time over the warp's lanes; of requests that end they are read, before a later step gives their
    // blocks to somebody else.
    const bool mine = q < p.n && (int)(q % gridDim.x) == (int)blockIdx.x && (back || (granted && need));
    for (unsigned todo = __ballot_sync(0xFFFFFFFFu, mine); todo; todo &= todo - 1) {
      const int from = __ffs((int)todo) - 1;
      const int nq = __shfl_sync(0xFFFFFFFFu, granted ? need : 0, from), bq = __shfl_sync(0xFFFFFFFFu, back, from);
      const int hq = __shfl_sync(0xFFFFFFFFu, have, from);
      const int take = head + __shfl_sync(0xFFFFFFFFu, upto - need, from);
      const long long give = (long long)head + count + __shfl_sync(0xFFFFFFFFu, (int)(sums >> 32) - back, from);
      int32_t* row = p.table + (long long)(q0 + (tid & ~31) + from) * p.ldt;
      for (int c = tid & 31; c < bq; c += 32) p.ring[(int)((give + c) % N)] = row[c];
      for (int c = tid & 31; c < nq; c += 32) row[hq + c] = p.ring[take + c >= N ? take + c - N : take + c];
    }
  }
  // granted requests that need blocks are the first of those that do, so the last of them has taken what all have
  taken = __reduce_max_sync(0xFFFFFFFFu, taken);
  refused = __reduce_add_sync(0xFFFFFFFFu, refused);
  __syncthreads();
  int* const most = reinterpret_cast<int*>(warps);
  if ((tid & 31) == 0) most[tid >> 5] = taken;
  __syncthreads();
  if (first) {
    if ((tid & 31) == 0 && refused) atomicAdd(p.status + 1, (uint32_t)refused);
    if (tid == 0) {
      for (int w = 1; w < kPlanThreads / 32; ++w) taken = max(taken, most[w]);
      const int back = (int)(blocks_before >> 32);
      p.row_start[0] = 0;
      p.state_out[0] = head + taken >= N ? head + taken - N : head + taken;
      p.state_out[1] = min(N, count - taken + back);
      if (count - taken + back > N) atomicAdd(p.status + 1, 1u);
    }
  }
  const int r0 = (int)((long long)p.rows * blockIdx.x / gridDim.x), r1 = (int)((long long)p.rows * (blockIdx.x + 1) / gridDim.x);
  const int live = p.n ? ends[p.n - 1] : 0;
  for (int r = r0 + tid; r < r1; r += kPlanThreads) {
    int slot = -1, pos = 0;
    if (r < live) {
      int lo = 0, hi = p.n - 1;                    // the first request that ends behind the row
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > r) hi = mid;
        else lo = mid + 1;
      }
      const int held = p.held[lo];
      pos = held + r - (lo ? ends[lo - 1] : 0);
      if (base[lo] >= 0) {
        const int have = blocks_of(held), c = pos / kAttnBlock;
        int from = head + base[lo] + c - have;
        const int id = c < have ? p.table[(long long)lo * p.ldt + c] : p.ring[from >= N ? from - N : from];
        if ((unsigned)id < (unsigned)N) slot = id * kAttnBlock + pos % kAttnBlock;
        else atomicAdd(p.status + 1, 1u);
      }
    }
    p.slot[r] = slot;
    p.position[r] = pos;
  }
}

// ---- append ----------------------------------------------------------------------------------------------------
// A warp takes rows of one head of the cache with the query heads that go with it; a lane holds dim / 32 neighbouring elements, its
// rotation's partner is in another lane (half layout) or its own. Bound by the bytes of q, k and v: each is read once, but for the first
// token of a block, whose size decides the block's exponent: a warp whose rows have it outside of them reads it again (from L2).
constexpr int kAppendWarps = 8;

__device__ __forceinline__ uint32_t pack16(int hi, int lo) {       // both saturated to 16 bits
  uint32_t r;
  asm("cvt.pack.sat.s16.s32 %0, %1, %2;" : "=r"(r) : "r"(hi), "r"(lo));
  return r;
}
__device__ __forceinline__ int low16(uint32_t v) { return (int)(short)(v & 0xFFFFu); }
__device__ __forceinline__ int high16(uint32_t v) { return (int)v >> 16; }

// A lane's elements of a row, in 16 bits.
template <class X, int E, bool kVector>
__device__ __forceinline__ void load(const X* p, int (&x)[E]) {
  if (kVector && sizeof(X) * E >= 2) {
    if (sizeof(X) == 4) {
      if (E == 4) {
        const int4 v = *reinterpret_cast<const int4*>(p);
        x[0] = v.x; x[1 % E] = v.y; x[2 % E] = v.z; x[3 % E] = v.w;
      } else if (E == 2) {
        const int2 v = *reinterpret_cast<const int2*>(p);
        x[0] = v.x; x[1 % E] = v.y;
      } else {
        x[0] = (int)p[0];
      }
    } else if (E == 4) {
      const char4 v = *reinterpret_cast<const char4*>(p);
      x[0] = v.x; x[1 % E] = v.y; x[2 % E] = v.z; x[3 % E] = v.w;
    } else {
      const char2 v = *reinterpret_cast<const char2*>(p);
      x[0] = v.x; x[1 % E] = v.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = (int)p[i];
  }
  if (sizeof(X) == 4) {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = min(max(x[i], -32768), 32767);
  }
}

// Factors of a lane's elements and of their partners, in 2^-14 (1 and 0 where nothing is rotated), and where the partners are.
template <int E>
struct Rotation {
  int c[E], s[E], from;
};

template <int E, int kLayout>
__device__ __forceinline__ Rotation<E> rotation(const AttnArgs& a, int position, int lane) {
  Rotation<E> r;
  const int half = a.rot / 2, d0 = lane * E;
  r.from = kLayout == kRotaryHalf ? (d0 < half ? lane + half / E : lane - half / E) : E == 1 ? lane ^ 1 : lane;
  if (d0 >= a.rot) r.from = lane;
  const short2* t = a.rotary + (long long)position * half;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int d = d0 + i;
    r.c[i] = 16384;
    r.s[i] = 0;
    if (d < a.rot) {
      const bool low = kLayout == kRotaryHalf ? d < half : (d & 1) == 0;
      const short2 v = t[kLayout == kRotaryHalf ? (low ? d : d - half) : d >> 1];
      r.c[i] = v.x;
      r.s[i] = low ? -(int)v.y : (int)v.y;
    }
  }
  return r;
}

template <int E, int kLayout>
__device__ __forceinline__ void rotate(int (&x)[E], const Rotation<E>& r) {
  int o[E];
  if (kLayout == kRotaryHalf || E == 1) {
    if (E == 1) {
      o[0] = __shfl_sync(0xFFFFFFFFu, x[0], r.from);
    } else {
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const uint32_t v = __shfl_sync(0xFFFFFFFFu, pack16(x[(i + 1) % E], x[i]), r.from);
        o[i] = low16(v);
        o[(i + 1) % E] = high16(v);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = x[i ^ (E > 1 ? 1 : 0)];
  }
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] = (x[i] * r.c[i] + o[i] * r.s[i] + 8192) >> 14;
}

template <int E>
__device__ __forceinline__ int largest(const int (&x)[E]) {        // |x| over the warp
  int m = abs(x[0]);
#pragma unroll
  for (int i = 1; i < E; ++i) m = max(m, abs(x[i]));
  return __reduce_max_sync(0xFFFFFFFFu, m);
}

// The smallest e with amax (8 + headroom) <= 1016 2^e.
__device__ __forceinline__ int exponent(int amax, int headroom) {
  const int over = (amax * (8 + headroom) + 1015) / 1016;
  return over <= 1 ? 0 : 32 - __clz(over - 1);
}

// The elements in 8 bits, -127 .. 127, in a word's low bytes.
template <int E>
__device__ __forceinline__ uint32_t pack8(const int (&x)[E], int e) {
  const int half = (1 << e) >> 1;
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) r |= (uint32_t)(min(max((x[i] + half) >> e, -127), 127) & 255) << (8 * i);
  return r;
}

template <int E>
__device__ __forceinline__ void store8(int8_t* p, uint32_t v) {
  if (E == 4) *reinterpret_cast<uint32_t*>(p) = v;
  else if (E == 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)v;
  else *p = (int8_t)v;
}

template <class X, int E, int kLayout, bool kVector>
__global__ void __launch_bounds__(32 * kAppendWarps) append_kernel(const AttnArgs a, const CacheArgs c, const AppendArgs p, const int per_warp) {
  constexpr int D = 32 * E, kPitch = D + 4;
  extern __shared__ uint8_t v8[];                  // [rows of the tile][kPitch]: values, to be turned around
  __shared__ int slots[4 * kAppendWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tile = per_warp * kAppendWarps;
  const int h = blockIdx.y, row0 = blockIdx.x * tile, d0 = lane * E;
  const int slot_end = c.blocks * kAttnBlock;      // below 2^31: the binding of a cache sees to that
  int first_row = -1, first_k = 0, first_v = 0;    // the last first token of a block that was looked at: exponents
  for (int i = 0; i < per_warp; ++i) {
    const int t = warp * per_warp + i, row = row0 + t;
    int slot = -1;
    if (row < p.rows) {
      slot = p.slot[row];
      int pos = p.position[row];
      bool bad = (a.rot && (unsigned)pos >= (unsigned)a.positions) || slot < -1 || slot >= slot_end;
      if (bad && lane == 0 && h == 0) atomicAdd(a.status + 1, 1u);
      if (slot < 0 || slot >= slot_end) slot = -1;
      pos = min(max(pos, 0), a.positions - 1);
      const Rotation<E> rot = rotation<E, kLayout>(a, pos, lane);
      const X* kr = (const X*)p.k + row * p.ldk + h * D + d0;
      const X* vr = (const X*)p.v + row * p.ldv + h * D + d0;
      int k[E], v[E];
      load<X, E, kVector>(kr, k);
      load<X, E, kVector>(vr, v);
      for (int g = 0; g < a.group; ++g) {
        const int head = h * a.group + g;
        int q[E];
        load<X, E, kVector>((const X*)p.q + row * p.ldq + head * D + d0, q);
        rotate<E, kLayout>(q, rot);
        const int e = exponent(largest<E>(q), 0);
        store8<E>(p.q8 + ((long long)row * a.heads + head) * D + d0, pack8<E>(q, e));
        if (lane == 0) p.q_exp[(long long)row * a.heads + head] = (uint8_t)e;
      }
      if (slot >= 0) {
        rotate<E, kLayout>(k, rot);
        const int off = slot % kAttnBlock, from = row - off;
        const long long at = (long long)(slot / kAttnBlock) * a.kv + h;
        int ek, ev;
        if (off == 0) {
          ek = exponent(largest<E>(k), a.k_headroom);
          ev = exponent(largest<E>(v), a.v_headroom);
          if (lane == 0) {
            c.k_exp[at] = (uint8_t)ek;
            c.v_exp[at] = (uint8_t)ev;
          }
        } else if (from >= 0 && (from == first_row || p.slot[from] == slot - off)) {
          if (from != first_row) {
            int f[E];
            load<X, E, kVector>((const X*)p.v + from * p.ldv + h * D + d0, f);
            first_v = exponent(largest<E>(f), a.v_headroom);
            load<X, E, kVector>((const X*)p.k + from * p.ldk + h * D + d0, f);
            rotate<E, kLayout>(f, rotation<E, kLayout>(a, min(max(p.position[from], 0), a.positions - 1), lane));
            first_k = exponent(largest<E>(f), a.k_headroom);
            first_row = from;
          }
          ek = first_k;
          ev = first_v;
        } else {
          ek = min((int)c.k_exp[at], kAttnMaxExp);
          ev = min((int)c.v_exp[at], kAttnMaxExp);
        }
        store8<E>(c.k + (at * kAttnBlock + off) * D + d0, pack8<E>(k, ek));
        const uint32_t w = pack8<E>(v, ev);
#pragma unroll
        for (int j = 0; j < E; ++j) v8[t * kPitch + d0 + j] = (uint8_t)(w >> (8 * j));
      }
    }
    if (lane == 0) slots[t] = slot;
  }
  __syncthreads();
  // values of four neighbouring tokens of a dimension lie side by side
  for (int i = threadIdx.x; i < tile / 4 * D; i += 32 * kAppendWarps) {
    const int t = i % (tile / 4) * 4, d = i / (tile / 4);
    const int s = slots[t];
    int8_t* out = c.v + ((long long)(s / kAttnBlock) * a.kv + h) * D * kAttnBlock + d * kAttnBlock + s % kAttnBlock;
    if (s >= 0 && s % 4 == 0 && slots[t + 1] == s + 1 && slots[t + 2] == s + 2 && slots[t + 3] == s + 3) {
      *reinterpret_cast<uint32_t*>(out) = v8[t * kPitch + d] | v8[(t + 1) * kPitch + d] << 8 | v8[(t + 2) * kPitch + d] << 16 |
                                          (uint32_t)v8[(t + 3) * kPitch + d] << 24;
    } else {
      for (int j = 0; j < 4; ++j) {
        const int sj = slots[t + j];
        if (sj >= 0)
          c.v[((long long)(sj / kAttnBlock) * a.kv + h) * D * kAttnBlock + d * kAttnBlock + sj % kAttnBlock] = (int8_t)v8[(t + j) * kPitch + d];
      }
    }
  }
}

template <class X, int E, int kLayout>
cudaError_t launch_append(const AttnArgs& a, const CacheArgs& c, const AppendArgs& p, cudaStream_t stream) {
  // four rows to a warp where that still leaves two CTAs to an SM
  const int per_warp = (long long)p.rows * a.kv >= 2ll * a.sms * 4 * kAppendWarps ? 4 : 1, tile = per_warp * kAppendWarps;
  const dim3 grid((unsigned)((p.rows + tile - 1) / tile), (unsigned)a.kv);
  const size_t smem = (size_t)tile * (32 * E + 4);
  if (p.vector) append_kernel<X, E, kLayout, true><<<grid, 32 * kAppendWarps, smem, stream>>>(a, c, p, per_warp);
  else append_kernel<X, E, kLayout, false><<<grid, 32 * kAppendWarps, smem, stream>>>(a, c, p, per_warp);
  return cudaGetLastError();
}

template <class X, int kLayout>
cudaError_t launch_append(const AttnArgs& a, const CacheArgs& c, const AppendArgs& p, cudaStream_t stream) {
  return a.dim == 128 ? launch_append<X, 4, kLayout>(a, c, p, stream)
                      : a.dim == 64 ? launch_append<X, 2, kLayout>(a, c, p, stream) : launch_append<X, 1, kLayout>(a, c, p, stream);
}

}  // namespace

cudaError_t launch_attn_plan(const PlanArgs& p, int sms, cudaStream_t stream) {
  const size_t smem = 8 * (size_t)p.n;
  const int grid = std::min(sms, std::max(1, std::max((p.rows + kPlanRows - 1) / kPlanRows, (p.n + 127) / 128)));
  plan_kernel<<<grid, kPlanThreads, smem, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t configure_attn_cache() {
  return cudaFuncSetAttribute(plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 8 * kAttnMaxRequests);
}

cudaError_t launch_attn_append(const AttnArgs& a, const CacheArgs& c, const AppendArgs& p, cudaStream_t stream) {
  if (a.x_i8)
    return a.layout == kRotaryInterleaved ? launch_append<int8_t, kRotaryInterleaved>(a, c, p, stream)
                                          : launch_append<int8_t, kRotaryHalf>(a, c, p, stream);
  return a.layout == kRotaryInterleaved ? launch_append<int, kRotaryInterleaved>(a, c, p, stream) : launch_append<int, kRotaryHalf>(a, c, p, stream);
}

}  // namespace iodf
