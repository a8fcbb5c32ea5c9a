// Norms before and after a block with its gate and residual scale (include/iodf.h: iodf_norm_forward).
//
// One pass: T threads hold a row of C channels in registers, E values each, from the loads to the stores; only the
// sums of a norm (sum, sum of squares) cross threads. What bounds it is memory, so every operand is loaded before
// the first value is used and the arithmetic is kept below the loads' time: per element and norm a square, and
// two 32 x 32 -> 64 multiply-adds whose rounding constant is the addend and of whose result only the high word is
// shifted. Three ways to lay a row over its threads:
//   kVector  eight neighbouring channels per thread, 8 or 16-byte accesses (everything aligned to them)
//   kScalar  neighbouring threads take neighbouring channels, one element per access (any alignment)
//   kPlanes  the residual stream as planes: as kScalar with T = 1 or 8, so that neighbouring threads take
//            neighbouring pixels of a plane (T = 8: four pixels of eight planes per warp and access)
#include <algorithm>
#include <type_traits>

#include "norm_kernel.h"
#include "../../include/iodf.h"

namespace iodf {
namespace {

enum { kVector = 0, kScalar = 1, kPlanes = 2 };

struct None {};

__device__ __forceinline__ int clip24(int v) { return min(max(v, -(1 << 23)), (1 << 23) - 1); }

// a b + c, its high word
__device__ __forceinline__ int mad_hi(int a, int b, long long c) { return (int)(((long long)a * b + c) >> 32); }

// What scales a row: N(v) = (v rho + 2^(sh-1)) >> sh, rho / 2^sh ~ 2^22 / sqrt(D), 1 <= D < 2^62, 9 <= sh <= 39. Where
// sh < 32 the values are small (|v| <= sqrt(D)): they are shifted up by 32 - sh first and stay below
// 2^24, so that the result is always the high word, shifted.
struct RowScale {
  int rho, up, down;
  long long round;
  __device__ __forceinline__ int operator()(int v) const { return mad_hi(v << up, rho, round) >> down; }
};

// sigma = floor(sqrt(m)) and rho = floor((2^61 - 1) / sigma) for m = D 2^t in [2^60, 2^62). Both come from one
// reciprocal root y in double precision. m y is off by less than 2^-19, so sigma is off by one at most;
// 1 / sigma = y (1 + e + e^2 ..) with e = (sqrt(m) - sigma) / sigma < 2^-30, whose square moves rho by less than 2^-28, so
// rho is off by one at most too. Both are put right in integers.
__device__ __forceinline__ RowScale row_scale(unsigned long long D) {
  const int t = (__clzll((long long)D) - 2) & ~1;
  const unsigned long long m = D << t;
  const double md = (double)m, y = rsqrt(md), root = md * y;
  unsigned int s = (unsigned int)fmin(root, 2147483647.0);
  if ((unsigned long long)s * s > m) --s;
  if ((unsigned long long)(s + 1) * (s + 1) <= m) ++s;
  const double e = (root - (double)s) * y;
  const unsigned long long top = (1ull << 61) - 1;
  unsigned int q = (unsigned int)fmin((y + y * e) * 2305843009213693952.0, 2147483647.0);
  if ((unsigned long long)q * s > top) --q;
  if ((unsigned long long)(q + 1) * s <= top) ++q;
  const int sh = 39 - (t >> 1);
  RowScale r;
  r.rho = (int)q;
  r.up = max(32 - sh, 0);
  r.down = max(sh - 32, 0);
  r.round = 1ll << (31 + r.down);
  return r;
}

// Sum over the T threads of a row of values 0 <= v < 2^54 / T (squares) or |v| < 2^47 / T (sums): in a whole warp two
// 32-bit reductions, of 27 low bits (16 for signed values) and of the rest.
template <int T, bool kSigned>
__device__ __forceinline__ long long row_sum(long long v, long long* red) {
  if constexpr (T == 1) return v;
  if constexpr (T < 32) {
#pragma unroll
    for (int o = T / 2; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
  } else {
    constexpr int kLow = kSigned ? 16 : 27;
    const unsigned int lo = __reduce_add_sync(0xFFFFFFFFu, (unsigned int)v & ((1u << kLow) - 1));
    const int hi = __reduce_add_sync(0xFFFFFFFFu, (int)(v >> kLow));
    long long s = kSigned ? ((long long)hi << kLow) + lo : ((long long)(unsigned int)hi << kLow) + lo;
    if constexpr (T > 32) {
      if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
      __syncthreads();
      s = 0;
#pragma unroll
      for (int w = 0; w < T / 32; ++w) s += red[w];
    }
    return s;
  }
}

// N over a row in registers; values behind the last channel are zero and stay so. red: kRedSlots sums of this norm
// (each sum has its own words, so one barrier per sum is enough).
template <int T, int E, class Valid>
__device__ __forceinline__ void norm_row(int (&v)[E], int C, int kind, unsigned long long eps, long long* red, Valid valid) {
  if (kind == IODF_NORM_CENTRED) {
    int s = 0;                                          // |s| <= 32 * 2^23
#pragma unroll
    for (int e = 0; e < E; ++e) s += v[e];
    const long long n = 2 * row_sum<T, true>(s, red) + C;
    // n / 2C is at least 1 / 2C = 2^-14 away from an integer that it is not, and below 2^24: floor of the rounded quotient
    const int mean = (int)floor((double)n / (double)(2 * C));
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = valid(e) ? v[e] - mean : 0;
  }
  long long q = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) q += (long long)v[e] * v[e];
  const RowScale scale = row_scale((unsigned long long)row_sum<T, false>(q, red + 16) + eps);
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = scale(v[e]);
}

// ---- eight neighbouring elements --------------------------------------------------------------------------
__device__ __forceinline__ void load8(const int* p, int (&v)[8]) {
  const int4 a = reinterpret_cast<const int4*>(p)[0], b = reinterpret_cast<const int4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const int16_t* p, int (&v)[8]) {
  const int4 a = *reinterpret_cast<const int4*>(p);
  const int w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = (int16_t)w[i];
    v[2 * i + 1] = w[i] >> 16;
  }
}
__device__ __forceinline__ void load8(const int8_t* p, int (&v)[8]) {
  const int2 a = *reinterpret_cast<const int2*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = (int8_t)(a.x >> (8 * i));
    v[4 + i] = (int8_t)(a.y >> (8 * i));
  }
}
__device__ __forceinline__ void load8(const uint8_t* p, int (&v)[8]) {
  const uint2 a = *reinterpret_cast<const uint2*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = (a.x >> (8 * i)) & 255;
    v[4 + i] = (a.y >> (8 * i)) & 255;
  }
}
__device__ __forceinline__ void store8(int* p, const int (&v)[8]) {
  reinterpret_cast<int4*>(p)[0] = make_int4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<int4*>(p)[1] = make_int4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(int16_t* p, const int (&v)[8]) {
  int w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __byte_perm(v[2 * i], v[2 * i + 1], 0x5410);
  *reinterpret_cast<int4*>(p) = make_int4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(uint8_t* p, const int (&v)[8]) {
  int2 a;
  a.x = __byte_perm(__byte_perm(v[0], v[1], 0x0040), __byte_perm(v[2], v[3], 0x0040), 0x5410);
  a.y = __byte_perm(__byte_perm(v[4], v[5], 0x0040), __byte_perm(v[6], v[7], 0x0040), 0x5410);
  *reinterpret_cast<int2*>(p) = a;
}

template <int T>
struct Block { static constexpr int threads = T <= 32 ? 128 : T, rows = threads / T; };

template <class RT, class BT, int T, int E, int MODE>
__global__ void __launch_bounds__(Block<T>::threads) norm_kernel(const NormArgs a) {
  constexpr bool kBlock = !std::is_same<BT, None>::value;
  using B = typename std::conditional<kBlock, BT, int8_t>::type;
  __shared__ long long red[64];
  constexpr int kRows = Block<T>::rows;
  const int t = threadIdx.x % T;
  const unsigned int row0 = blockIdx.x * kRows + threadIdx.x / T, rows = (unsigned int)a.rows;
  // a row beyond the last one is computed again by the spare threads of a warp (they take part in its reductions) and not stored
  const bool live = row0 < rows;
  const unsigned int row = live ? row0 : rows - 1;
  const int C = a.channels;
  auto channel = [&](int e) { return MODE == kVector ? ((e / 8) * T + t) * 8 + e % 8 : e * T + t; };
  auto valid = [&](int e) { return channel(e) < C; };

  const RT* rp;
  RT* op = nullptr;
  if (MODE == kPlanes) {
    const unsigned int rpx = (unsigned int)a.rv.pixels, opx = (unsigned int)a.ov.pixels;
    rp = (const RT*)a.r + (long long)(row / rpx) * a.rv.img + (long long)(row % rpx) * a.rv.pix;
    if (kBlock) op = (RT*)a.r_out + (long long)(row / opx) * a.ov.img + (long long)(row % opx) * a.ov.pix;
  } else {
    rp = (const RT*)a.r + (long long)row * a.rv.pix;
    if (kBlock) op = (RT*)a.r_out + (long long)row * a.ov.pix;
  }
  const long long rc = MODE == kPlanes ? a.rv.chan : 1, oc = MODE == kPlanes ? a.ov.chan : 1;
  const B* bp = (const B*)a.b + (long long)row * a.ldb;
  const uint8_t* gp = a.gate + (long long)row * a.ldg;
  uint8_t* np = (uint8_t*)a.n + (long long)row * a.ldn;

  int v[E], r[E];
  if (MODE == kVector) {
#pragma unroll
    for (int i = 0; i < E / 8; ++i) {
      const int c = channel(8 * i);
      int x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (c + 8 <= C) {
        load8(rp + c, x);
        if (kBlock) load8(bp + c, y);
      } else if (c < C) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < C) {
            x[e] = rp[c + e];
            if (kBlock) y[e] = bp[c + e];
          }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        r[8 * i + e] = x[e];
        v[8 * i + e] = y[e];
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      r[e] = valid(e) ? rp[channel(e) * rc] : 0;
      v[e] = kBlock && valid(e) ? bp[channel(e)] : 0;
    }
  }
  if (sizeof(RT) == 4)
#pragma unroll
    for (int e = 0; e < E; ++e) r[e] = clip24(r[e]);

  if constexpr (kBlock) {
    if (sizeof(B) == 4)
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = clip24(v[e]);
    if (a.post) norm_row<T>(v, C, a.post, a.eps, red, valid);
    const long long round = 1ll << (30 + a.shift);
    if (MODE == kVector) {
#pragma unroll
      for (int i = 0; i < E / 8; ++i) {
        const int c = channel(8 * i);
        if (c >= C) continue;
        int m[8], g[8], o[8];
        load8(a.mult + c, m);
        if (a.gate) {
          if (c + 8 <= C) {
            load8(gp + c, g);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = c + e < C ? gp[c + e] : 0;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) v[8 * i + e] *= g[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
          o[e] = min(max(r[8 * i + e] + (mad_hi(v[8 * i + e], m[e], round) >> (a.shift - 1)), a.res_lo), a.res_hi);
        if (c + 8 <= C) {
          if (live) store8(op + c, o);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (live && c + e < C) op[c + e] = (RT)o[e];
            if (c + e >= C) o[e] = 0;                   // the clip's range need not hold zero
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) r[8 * i + e] = o[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (valid(e)) {
          const int c = channel(e);
          if (a.gate) v[e] *= gp[c];
          r[e] = min(max(r[e] + (mad_hi(v[e], a.mult[c], round) >> (a.shift - 1)), a.res_lo), a.res_hi);
          if (live) op[c * oc] = (RT)r[e];
        }
    }
  }

  if (a.pre) {
    norm_row<T>(r, C, a.pre, a.eps, red + 32, valid);
    const long long round = 1ll << (30 + a.n_shift);
    if (MODE == kVector) {
#pragma unroll
      for (int i = 0; i < E / 8; ++i) {
        const int c = channel(8 * i);
        if (c >= C) continue;
        int m[8], o[8], d[8];
        load8(a.n_mult + c, m);
        load8(a.n_bias + c, d);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          o[e] = min(max((mad_hi(r[8 * i + e], m[e], round) >> (a.n_shift - 1)) + d[e], a.n_lo), a.n_hi);
        if (!live) continue;
        if (c + 8 <= C) {
          store8(np + c, o);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + e < C) np[c + e] = (uint8_t)o[e];
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (live && valid(e)) {
          const int c = channel(e);
          np[c] = (uint8_t)min(max((mad_hi(r[e], a.n_mult[c], round) >> (a.n_shift - 1)) + a.n_bias[c], a.n_lo), a.n_hi);
        }
    }
  }
}

template <class RT, class BT, int T, int E, int MODE>
cudaError_t run(const NormArgs& a, cudaStream_t stream) {
  constexpr int kRows = Block<T>::rows;
  norm_kernel<RT, BT, T, E, MODE><<<(unsigned int)((a.rows + kRows - 1) / kRows), Block<T>::threads, 0, stream>>>(a);
  return cudaGetLastError();
}

bool vectors(const void* p, long long ld, int size) {   // rows of eight elements in 8 or 16-byte accesses
  const int n = size == 1 ? 8 : 16;
  return !p || (reinterpret_cast<uintptr_t>(p) % n == 0 && ld * size % n == 0);
}

template <class RT, class BT>
cudaError_t pick(NormArgs a, cudaStream_t stream) {
  constexpr int kB = std::is_same<BT, None>::value ? 1 : (int)sizeof(BT);
  const int C = a.channels;
  // a view whose images follow each other without a gap is rows
  const bool rows = a.rv.chan == 1 && (!a.has_block || a.ov.chan == 1) && a.rv.pixels >= a.rows && (!a.has_block || a.ov.pixels >= a.rows);
  if (!rows) {
    a.rv.pixels = std::min(a.rv.pixels, 0xFFFFFFFFll);
    a.ov.pixels = a.has_block ? min(a.ov.pixels, 0xFFFFFFFFll) : 1;
    if (C <= 8) return run<RT, BT, 1, 8, kPlanes>(a, stream);
    if (C <= 32) return run<RT, BT, 1, 32, kPlanes>(a, stream);
    if (C <= 128) return run<RT, BT, 8, 16, kPlanes>(a, stream);
    if (C <= 256) return run<RT, BT, 8, 32, kPlanes>(a, stream);
    if (C <= 2048) return run<RT, BT, 128, 16, kPlanes>(a, stream);
    return run<RT, BT, 512, 16, kPlanes>(a, stream);
  }
  if (vectors(a.r, a.rv.pix, sizeof(RT)) && vectors(a.r_out, a.ov.pix, sizeof(RT)) && vectors(a.b, a.ldb, kB) &&
      vectors(a.gate, a.ldg, 1) && vectors(a.n, a.ldn, 1)) {
    if (C <= 64) return run<RT, BT, 8, 8, kVector>(a, stream);
    if (C <= 128) return run<RT, BT, 16, 8, kVector>(a, stream);
    if (C <= 256) return run<RT, BT, 32, 8, kVector>(a, stream);
    if (C <= 512) return run<RT, BT, 32, 16, kVector>(a, stream);
    if (C <= 1024) return run<RT, BT, 64, 16, kVector>(a, stream);
    if (C <= 2048) return run<RT, BT, 128, 16, kVector>(a, stream);
    if (C <= 4096) return run<RT, BT, 256, 16, kVector>(a, stream);
    return run<RT, BT, 512, 16, kVector>(a, stream);
  }
  if (C <= 64) return run<RT, BT, 8, 8, kScalar>(a, stream);
  if (C <= 256) return run<RT, BT, 32, 8, kScalar>(a, stream);
  if (C <= 512) return run<RT, BT, 32, 16, kScalar>(a, stream);
  if (C <= 2048) return run<RT, BT, 128, 16, kScalar>(a, stream);
  return run<RT, BT, 512, 16, kScalar>(a, stream);
}

template <class RT>
cudaError_t pick_block(const NormArgs& a, cudaStream_t stream) {
  if (!a.has_block) return pick<RT, None>(a, stream);
  return a.block_i8 ? pick<RT, int8_t>(a, stream) : pick<RT, int32_t>(a, stream);
}

}  // namespace

cudaError_t launch_norm(const NormArgs& a, cudaStream_t stream) {
  return a.res_i16 ? pick_block<int16_t>(a, stream) : pick_block<int32_t>(a, stream);
}

}  // namespace iodf
