// Norms before and after a block with its gate and residual scale (include/iodf.h: iodf_norm_forward).
//
// One pass: T threads hold a row of C channels in registers, E values each, from the loads to the stores; only the
// sums of a norm (sum, sum of squares) cross threads. Every operand is loaded before the first value is used.
// What bounds it: memory where the arithmetic stays below it. An element costs a 64-bit square (some 5 clocks per warp and
// SM quarter), per norm two 32 x 32 -> 64 multiply-adds (5 each) and a shift of the pair (2), clips and packs; a row costs some
// 250 instructions per thread beside its elements. 16384 x 4096 int16 with int32 blocks and gates: 134 us (5.0 TB/s; floor 104;
// without the two norms 87), 32768 x 256 int32 with int8 blocks: 20.9 us (4.0 TB/s; floor 13), 20011 x 173 unaligned,
// centred: 19.2 us (2.5 TB/s; floor 7.5; a row's own work), one row of 4096: 4 us (a launch).
// Measured and not taken, on the first of these while it took 182 us (its loads still stood behind guards, so these say nothing of the
// present form): 32 elements per thread 228 us (a fifth of the warps), rows copied ahead into shared memory 235 (twice through the same
// pipe), a row's two roots worked out by one thread for all 188 (two more barriers), four elements per access 222.
// Three ways to lay a row over its threads:
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

// What scales a row: N(v) = (v rho + 2^(sh-1)) >> sh, rho / 2^sh ~ 2^22 / sqrt(D), 1 <= D < 2^62, 9 <= sh <= 39.
struct RowScale {
  int rho, sh;
  long long round;
};

// sigma = floor(sqrt(m)) and rho = floor((2^61 - 1) / sigma) for m = D 2^t in [2^60, 2^62). Both come from one
// reciprocal root y of m: the hardware's estimate (more than 20 bits) and one step of third order, whose error (5/16 e^3 and
// roundings, together below 2^-50) puts m y and 2^61 y (1 + e') within 2^-18 of the root and the quotient; e' = (root - sigma) y
// < 2^-30 and its square, below 2^-60, moves rho by less than 2^-28. Rounded to integers by adding 1.5 * 2^52,
// sigma is the floor or one more; rho belongs to that integer and is up to three less for the one below it. Exact remainders put
// both right.
__device__ __forceinline__ RowScale row_scale(unsigned long long D) {
  constexpr double kMagic = 6755399441055744.0;         // 1.5 * 2^52: the low word of the sum is the nearest integer
  const int t = (__clzll((long long)D) - 2) & ~1;
  const unsigned long long m = D << t;
  const double md = (double)m;
  double y;
  asm("rsqrt.approx.ftz.f64 %0, %1;" : "=d"(y) : "d"(md));
  const double h = fma(-md * y, y, 1.0);
  y = fma(y * h, fma(h, 0.375, 0.5), y);
  const double root = md * y, rs = root + kMagic;
  unsigned int s = (unsigned int)__double2loint(rs);
  long long rem = (long long)(m - (unsigned long long)s * s);          // 0 .. 2 s if s is the floor
  const double e = (root - (rs - kMagic)) * y;
  unsigned int q = (unsigned int)__double2loint(fma(fma(y, e, y), 2305843009213693952.0, kMagic));
  // s too large by one: rem < 0; too small: rem > 2 s
  const int ds = rem < 0 ? -1 : rem > 2ll * s ? 1 : 0;
  s += ds;
  rem = (long long)(((1ull << 61) - 1) - (unsigned long long)q * s);   // 0 .. s - 1 if q is the floor
  while (rem < 0) { --q; rem += s; }
  while (rem >= (long long)s) { ++q; rem -= s; }
  RowScale r;
  r.rho = (int)q;
  r.sh = 39 - (t >> 1);
  r.round = 1ll << (r.sh - 1);
  return r;
}

// Sum over the T threads of a row. In a whole warp two 32-bit reductions, of 27 low bits (16 for signed values) and of the rest,
// which hold values of a thread 0 <= v < 2^54 (squares; 16 centred values are at most 2^52) and |v| < 2^42 (sums; at most 2^27).
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
      s = red[threadIdx.x & (T / 32 - 1)];
#pragma unroll
      for (int o = T / 64; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
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
  const RowScale s = row_scale((unsigned long long)row_sum<T, false>(q, red + 16) + eps);
  if (s.sh < 32) {                                      // sqrt(D) below 2^23: a funnel shift of the two words
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const long long p = (long long)v[e] * s.rho + s.round;
      v[e] = (int)__funnelshift_r((unsigned int)p, (unsigned int)(p >> 32), s.sh);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = mad_hi(v[e], s.rho, s.round) >> (s.sh - 32);
  }
}

// ---- eight neighbouring elements, as they lie in memory until they are used --------------------------------------
template <class Q>
struct Raw8 {
  uint32_t w[2 * sizeof(Q)];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (int)(2 * sizeof(Q)); ++i) w[i] = 0;
  }
  __device__ __forceinline__ void load(const Q* p) {
    if (sizeof(Q) == 1) {
      const uint2 a = *reinterpret_cast<const uint2*>(p);
      w[0] = a.x; w[1] = a.y;
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(Q) / 2; ++i) {
        const uint4 a = reinterpret_cast<const uint4*>(p)[i];
        w[4 * i] = a.x; w[4 * i + 1] = a.y; w[4 * i + 2] = a.z; w[4 * i + 3] = a.w;
      }
    }
  }
  __device__ __forceinline__ int at(int e) const {
    if (sizeof(Q) == 4) return (int)w[e];
    if (sizeof(Q) == 2) return e & 1 ? (int)w[e / 2] >> 16 : (int)(int16_t)w[e / 2];
    if (Q(-1) < Q(0)) return (int)(int8_t)(w[e / 4] >> (8 * (e & 3)));
    return (int)((w[e / 4] >> (8 * (e & 3))) & 255u);
  }
};
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
// clip to the whole range of int8 or uint8
__device__ __forceinline__ void store8_sat(uint8_t* p, const int (&v)[8], bool is_signed) {
  uint32_t w[2], t;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (is_signed) {
      asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(t) : "r"(v[4 * i + 3]), "r"(v[4 * i + 2]), "r"(0));
      asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(w[i]) : "r"(v[4 * i + 1]), "r"(v[4 * i]), "r"(t));
    } else {
      asm("cvt.pack.sat.u8.s32.b32 %0, %1, %2, %3;" : "=r"(t) : "r"(v[4 * i + 3]), "r"(v[4 * i + 2]), "r"(0));
      asm("cvt.pack.sat.u8.s32.b32 %0, %1, %2, %3;" : "=r"(w[i]) : "r"(v[4 * i + 1]), "r"(v[4 * i]), "r"(t));
    }
  }
  *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}

template <int T>
struct Block { static constexpr int threads = T <= 32 ? 128 : T, rows = threads / T; };

// Blocks per SM that the registers have to leave room for: what measured best (32 to 40 warps). It costs up to 64 bytes of spills in the
// forms with int32 residuals (T = 256; 32 for T = 128, 8 to 56 for unaligned rows of 161 to 256 channels), up to 44 with int16. us without
// and with the bound: 16384 x 4096 int16, int32 blocks, gates 153 and 134; int32 residuals, gates: 8192 x 8192, int8 blocks 238 and 174;
// 16384 x 4096, int8 160 and 158, int32 171 and 177 (spills); 32768 x 2048, int8 145 and 140, int32 156
// and 152; 65536 x 1024, int8 141 and 135; 131072 x 256, int8 74 and 70; unaligned, 100003 rows, int32: 173 channels 73 and 72, 199 78
// and 80, 225 86 and 86, 249 87 and 87.
template <int T, int E, int MODE>
__host__ __device__ constexpr int min_blocks() {
  return MODE == kScalar ? (T == 32 && E <= 8 ? 10 : 1) : MODE != kVector ? 1 : T == 512 ? 2 : T == 256 ? 5 : T == 128 ? 9 : T == 64 ? 16 : E <= 8 ? 10 : 8;
}

template <class RT, class BT, int T, int E, int MODE, bool kFull>
__global__ void __launch_bounds__(Block<T>::threads, min_blocks<T, E, MODE>()) norm_kernel(const NormArgs a) {
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
  auto valid = [&](int e) {
    if (kFull) return MODE == kVector || e < E - 1 || channel(e) < C;
    return channel(e) < C;
  };

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

  // Every operand of the row is asked for here, before the first is used. kVector has whole vectors only (C is a
  // multiple of 8), and with kFull every thread has its E channels (kScalar: all but the last), so that no guard stands between
  // the tables' loads either: a guarded load waits by itself (measured: a gate of 67 MB cost 50 us so, 8 us now).
  int v[E], r[MODE == kVector ? 1 : E];
  Raw8<RT> rr[MODE == kVector ? E / 8 : 1];
  Raw8<uint8_t> gr[MODE == kVector ? E / 8 : 1];
  int g[MODE == kVector ? 1 : E];
  const bool gated = kBlock && a.gate != nullptr;
  if constexpr (MODE == kVector) {
    Raw8<B> br[E / 8];
#pragma unroll
    for (int i = 0; i < E / 8; ++i) {
      const int c = channel(8 * i);
      if (!kFull) {
        rr[i].zero();
        br[i].zero();
      }
      if (kFull || c < C) {
        rr[i].load(rp + c);
        if (kBlock) br[i].load(bp + c);
        if (gated) gr[i].load(gp + c);
      }
    }
    if (kBlock) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = sizeof(B) == 4 ? clip24(br[e / 8].at(e % 8)) : br[e / 8].at(e % 8);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      r[e] = valid(e) ? rp[channel(e) * rc] : 0;
      v[e] = kBlock && valid(e) ? bp[channel(e)] : 0;
    }
    if (gated) {
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] = valid(e) ? gp[channel(e)] : 0;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (sizeof(RT) == 4) r[e] = clip24(r[e]);
      if (kBlock && sizeof(B) == 4) v[e] = clip24(v[e]);
    }
  }
  auto residual = [&](int e) {
    if constexpr (MODE != kVector) {
      return r[e];
    } else {
      const int x = rr[e / 8].at(e % 8);
      return sizeof(RT) == 4 ? clip24(x) : x;
    }
  };

  if constexpr (kBlock) {
    if (a.post) norm_row<T>(v, C, a.post, a.eps, red, valid);
    const long long round = 1ll << (30 + a.shift);
    if constexpr (MODE == kVector) {
#pragma unroll
      for (int i = 0; i < E / 8; ++i) {
        const int c = channel(8 * i);
        if (kFull || c < C) {
          Raw8<int> m;
          m.load(a.mult + c);
          int o[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int u = gated ? v[8 * i + e] * gr[i].at(e) : v[8 * i + e];
            o[e] = min(max(residual(8 * i + e) + (mad_hi(u, m.at(e), round) >> (a.shift - 1)), a.res_lo), a.res_hi);
          }
          if (live) store8(op + c, o);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[8 * i + e] = o[e];
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (valid(e)) {
          const int c = channel(e);
          if (gated) v[e] *= g[e];
          const int o = min(max(r[e] + (mad_hi(v[e], a.mult[c], round) >> (a.shift - 1)), a.res_lo), a.res_hi);
          if (live) op[c * oc] = (RT)o;
          v[e] = o;
        }
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = residual(e);
  }

  if (a.pre) {
    norm_row<T>(v, C, a.pre, a.eps, red + 32, valid);
    const long long round = 1ll << (30 + a.n_shift);
    if constexpr (MODE == kVector) {
#pragma unroll
      for (int i = 0; i < E / 8; ++i) {
        const int c = channel(8 * i);
        if (kFull || c < C) {
          Raw8<int> m, d;
          m.load(a.n_mult + c);
          d.load(a.n_bias + c);
          int o[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = (mad_hi(v[8 * i + e], m.at(e), round) >> (a.n_shift - 1)) + d.at(e);
          if (!a.n_full) {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = min(max(o[e], a.n_lo), a.n_hi);
          }
          if (live) store8_sat(np + c, o, a.n_lo < 0);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (live && valid(e)) {
          const int c = channel(e);
          np[c] = (uint8_t)min(max((mad_hi(v[e], a.n_mult[c], round) >> (a.n_shift - 1)) + a.n_bias[c], a.n_lo), a.n_hi);
        }
    }
  }
}

template <class RT, class BT, int T, int E, int MODE>
cudaError_t run(const NormArgs& a, cudaStream_t stream) {
  constexpr int kRows = Block<T>::rows;
  const unsigned int grid = (unsigned int)((a.rows + kRows - 1) / kRows);
  // every thread has E channels (kScalar: E - 1 and perhaps one more)
  const bool full = MODE == kVector ? a.channels == T * E : MODE == kScalar && a.channels > T * (E - 1);
  if (full) norm_kernel<RT, BT, T, E, MODE, MODE != kPlanes><<<grid, Block<T>::threads, 0, stream>>>(a);
  else norm_kernel<RT, BT, T, E, MODE, false><<<grid, Block<T>::threads, 0, stream>>>(a);
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
    a.ov.pixels = a.has_block ? std::min(a.ov.pixels, 0xFFFFFFFFll) : 1;
    if (C <= 8) return run<RT, BT, 1, 8, kPlanes>(a, stream);
    if (C <= 32) return run<RT, BT, 1, 32, kPlanes>(a, stream);
    if (C <= 128) return run<RT, BT, 8, 16, kPlanes>(a, stream);
    if (C <= 256) return run<RT, BT, 8, 32, kPlanes>(a, stream);
    if (C <= 2048) return run<RT, BT, 128, 16, kPlanes>(a, stream);
    return run<RT, BT, 512, 16, kPlanes>(a, stream);
  }
  if (C % 8 == 0 && vectors(a.r, a.rv.pix, sizeof(RT)) && vectors(a.r_out, a.ov.pix, sizeof(RT)) && vectors(a.b, a.ldb, kB) &&
      vectors(a.gate, a.ldg, 1) && vectors(a.n, a.ldn, 1)) {
    if (C <= 64) return run<RT, BT, 8, 8, kVector>(a, stream);
    if (C <= 128) return run<RT, BT, 16, 8, kVector>(a, stream);
    if (C <= 256) return run<RT, BT, 16, 16, kVector>(a, stream);
    if (C <= 512) return run<RT, BT, 32, 16, kVector>(a, stream);
    if (C <= 1024) return run<RT, BT, 64, 16, kVector>(a, stream);
    if (C <= 2048) return run<RT, BT, 128, 16, kVector>(a, stream);
    if (C <= 4096) return run<RT, BT, 256, 16, kVector>(a, stream);
    return run<RT, BT, 512, 16, kVector>(a, stream);
  }
  if (C <= 64) return run<RT, BT, 8, 8, kScalar>(a, stream);
  switch ((C + 31) / 32) {                              // of the widths that pruning leaves: only the last element is guarded
    case 3: return run<RT, BT, 32, 3, kScalar>(a, stream);
    case 4: return run<RT, BT, 32, 4, kScalar>(a, stream);
    case 5: return run<RT, BT, 32, 5, kScalar>(a, stream);
    case 6: return run<RT, BT, 32, 6, kScalar>(a, stream);
    case 7: return run<RT, BT, 32, 7, kScalar>(a, stream);
    case 8: return run<RT, BT, 32, 8, kScalar>(a, stream);
  }
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
