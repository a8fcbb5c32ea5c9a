// The arithmetic of integer attention (include/iodf.h: iodf_attn_forward), as all of its kernels compute it.
#pragma once
#include <stdint.h>

#include "attn.h"

namespace iodf {

// Weights. 2^(n / 8192), n = t - T <= 0 in 2^-13 octaves: octave and segment of 2^-6 octaves come from n's bits, and within a segment
// the mantissa rises by 2^-13 a step, so that a float's bits are one table word plus 1024 n: subtracting octaves lowers
// its exponent. Segments are laid through the curve's middle in them (0.22 % off at most, 0.05 % on average), the first one through 1 (0.46 %).
// Mantissas in units of 2^-23, less 2^23: round(2^(23 + (2 c + 1) / 128)) - 2^16, at least 2^23.
constexpr int kWeightSegments = 64;
__device__ const int kSegments[kWeightSegments] = {
    0, 71855, 164697, 258550, 353425, 449333, 546286, 644294, 743370, 843524, 944769, 1047117,
    1150578, 1255167, 1360895, 1467773, 1575816, 1685035, 1795443, 1907054, 2019880, 2133935, 2249231, 2365784,
    2483605, 2602709, 2723110, 2844823, 2967860, 3092238, 3217970, 3345071, 3473556, 3603440, 3734738, 3867466,
    4001640, 4137275, 4274386, 4412991, 4553105, 4694744, 4837926, 4982668, 5128985, 5276895, 5426417, 5577566,
    5730361, 5884820, 6040962, 6198803, 6358363, 6519661, 6682715, 6847544, 7014169, 7182608, 7352881, 7525008,
    7699009, 7874906, 8052717, 8232465};
constexpr int kWeightLow = -(1 << 18);        // weights are 0 from -2^17 on

// The table word of segment c: bits of the float mantissa * 2^-8 at its start, less what 1024 n will add.
__device__ __forceinline__ int weight_word(int c) { return ((127 + 15) << 23) + kSegments[c] - c * (128 << 10); }

// 0 .. 32768, rounded to nearest even, plus 128; the float's low bits are the number.
__device__ __forceinline__ uint32_t weight_bits(int n, int word) {
  return __float_as_uint(__fadd_rn(__int_as_float(word + (n << 10)), 8388608.f + 128.f));
}
constexpr uint32_t kWeightBias = 0x4B000080u; // weight_bits of a weight of 0

// W = min(2^31 - 1, floor(m0 2^(eq + ek) / 2^s))
__device__ __forceinline__ int score_multiplier(uint32_t m0, int e, int s) {
  const unsigned long long w = ((unsigned long long)m0 << e) >> s;
  return (int)min(w, 0x7FFFFFFFull);
}

// t = floor(score W / 2^23): |score| < 2^21 (128 products of at most 127 * 127), so that it has nine bits of room
__device__ __forceinline__ int score_octaves(int score, int W) { return __mulhi(score << 9, W); }

// What the sums of a row's weights make of its sums of weighted values: o = A 2^(V + 8) / L in 2^-8 units of v.
struct Reciprocal {
  uint32_t rho;
  int a, V;
};
__device__ __forceinline__ Reciprocal reciprocal(long long L, int V) {
  Reciprocal r;
  r.V = V;
  r.a = __clzll(L) - 32;                       // 2^31 <= L 2^a < 2^32
  const unsigned long long l = r.a >= 0 ? (unsigned long long)L << r.a : (unsigned long long)L >> -r.a;
  // The quotient of doubles is off by less than one (it has 32 bits); the remainder says which way.
  constexpr unsigned long long kTop = 0x7FFFFFFFFFFFFFFFull;
  unsigned long long q = (unsigned long long)(9223372036854775808.0 * __drcp_rn((double)l));
  if (q * l > kTop) --q;
  else if (kTop - q * l >= l) ++q;
  r.rho = (uint32_t)q;
  return r;
}
// A = 256 hi + lo
__device__ __forceinline__ int quotient(int hi, int lo, const Reciprocal& r) {
  const long long A = (long long)hi * 65536 + (long long)lo * 256;                       // 2^8 A, so that the next shift is to the right
  const int scaled = (int)__funnelshift_r((uint32_t)A, (uint32_t)(A >> 32), (uint32_t)(16 - r.a));     // floor(A 2^(a - 8)): |A| <= 127 L, 31 bits
  const int top = __mulhi(scaled, (int)r.rho) + scaled;            // scaled rho / 2^32: rho has its highest bit, as an int it is 2^32 less
  return (top + ((1 << (15 - r.V)) >> 1)) >> (15 - r.V);
}

// floor((o M0 + 2^(30 + s)) / 2^(31 + s)), and its clip; out: {M0, s, low and high word of the addend}; |o| < 2^27
__device__ __forceinline__ int requantised(int o, int4 out) {
  const long long v = (long long)o * out.x + (long long)((unsigned long long)(uint32_t)out.w << 32 | (uint32_t)out.z);
  return (int)__funnelshift_l((uint32_t)v, (uint32_t)(v >> 32), 1) >> out.y;
}
__device__ __forceinline__ int clipped(int y, int lo, int hi) { return min(max(y, lo), hi); }

// Keys that a row sees: [first, last)
struct Range {
  int first, last;
};
__device__ __forceinline__ Range visible(const AttnArgs& a, int position, int held) {
  Range r;
  r.last = a.causal ? min(held, position + 1) : held;
  r.first = a.window ? max(0, position - a.window + 1) : 0;
  return r;
}

}  // namespace iodf
