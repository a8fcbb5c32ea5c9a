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
      if (count + back > N) atomicAdd(p.status + 1, 1u);
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
// A warp takes 128 neighbouring elements of a row of q, k or v at a time (one head of 128, two of 64, four of 32), a lane four of them; the
// rotation's partner is in another lane (half layout) or the lane's own. The bytes: q, k and v are read once, but for the first token of a
// block, whose size decides the block's exponent: a warp whose rows have it outside of them reads it again (from L2). Those of 32-bit inputs
// take more than half of the time (16384 rows of 32 query and 8 cache heads of 128: 136 us, 3.7 TB/s); of 8-bit inputs the instructions
// do, some hundred for 128 elements (20011 rows of 16 and 4 of 64, half of each rotated: 37.5 us, four fifths of the issue slots). The next
// chunk of q is on its way while one is rotated (51 us had become 46 by it, with six CTAs to an SM instead of eight). Values of a tile of rows
// go through shared memory to be turned around.
constexpr int kAppendWarps = 8;          // rows of a tile: as many, or four times that
constexpr int kChunk = 128, kPitch = kChunk + 4;

__device__ __forceinline__ uint32_t pack16(int hi, int lo) {       // both saturated to 16 bits
  uint32_t r;
  asm("cvt.pack.sat.s16.s32 %0, %1, %2;" : "=r"(r) : "r"(hi), "r"(lo));
  return r;
}
__device__ __forceinline__ int low16(uint32_t v) { return (int)(short)(v & 0xFFFFu); }
__device__ __forceinline__ int high16(uint32_t v) { return (int)v >> 16; }

// A lane's four elements: in 16 bits, two words of two, or in 8 bits as they come.
struct Four {
  uint32_t a, b;
};
struct Bytes {
  uint32_t w;
};

template <bool kVector>
__device__ __forceinline__ Four load(const int* p, bool live) {
  if (!live) return {0, 0};
  int x[4];
  if (kVector) {
    const int4 v = *reinterpret_cast<const int4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = p[i];
  }
  return {pack16(x[1], x[0]), pack16(x[3], x[2])};
}
template <bool kVector>
__device__ __forceinline__ Bytes load(const int8_t* p, bool live) {
  if (!live) return {0};
  if (kVector) return {*reinterpret_cast<const uint32_t*>(p)};
  return {(uint32_t)(uint8_t)p[0] | (uint32_t)(uint8_t)p[1] << 8 | (uint32_t)(uint8_t)p[2] << 16 | (uint32_t)(uint8_t)p[3] << 24};
}
__device__ __forceinline__ void unpack(const Four& v, int (&x)[4]) { x[0] = low16(v.a); x[1] = high16(v.a); x[2] = low16(v.b); x[3] = high16(v.b); }
__device__ __forceinline__ void unpack(const Bytes& v, int (&x)[4]) {
  const char4 c = *reinterpret_cast<const char4*>(&v.w);
  x[0] = c.x; x[1] = c.y; x[2] = c.z; x[3] = c.w;
}

// Factors of a lane's elements and of their partners, in 2^-14 (1 and 0 where nothing is rotated), and where the partners are. For 8-bit elements
// in one word, the partner's in its high half.
template <class X>
struct Rotation {
  int c[4], s[4], from;
};

template <class X, int D, int kLayout>
__device__ __forceinline__ Rotation<X> rotation(const AttnArgs& a, int position, int lane) {
  Rotation<X> r;
  const int half = a.rot / 2, d0 = lane * 4 % D;
  const bool turned = d0 < a.rot, low = d0 < half;
  r.from = kLayout == kRotaryHalf && turned ? (low ? lane + half / 4 : lane - half / 4) : lane;
  int4 cs = make_int4(16384, 16384, 16384, 16384);
  if (turned) {
    const short2* t = a.rotary + (long long)position * half;
    if (kLayout == kRotaryHalf) {
      cs = *reinterpret_cast<const int4*>(t + (low ? d0 : d0 - half));
    } else {
      const int2 v = *reinterpret_cast<const int2*>(t + d0 / 2);
      cs = make_int4(v.x, v.x, v.y, v.y);
    }
  }
  const uint32_t v[4] = {(uint32_t)cs.x, (uint32_t)cs.y, (uint32_t)cs.z, (uint32_t)cs.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool minus = kLayout == kRotaryHalf ? low : i % 2 == 0;
    if (sizeof(X) == 1) {
      r.c[i] = (int)(minus ? (v[i] & 0xFFFFu) | (0u - (v[i] & 0xFFFF0000u)) : v[i]);
      r.s[i] = 0;
    } else {
      r.c[i] = low16(v[i]);
      r.s[i] = minus ? -high16(v[i]) : high16(v[i]);
    }
  }
  return r;
}

template <int kLayout>
__device__ __forceinline__ void rotate(const Four& v, const Rotation<int>& r, bool any, int (&x)[4]) {
  unpack(v, x);
  if (!any) return;
  int o[4];
  if (kLayout == kRotaryHalf) {
    unpack(Four{__shfl_sync(0xFFFFFFFFu, v.a, r.from), __shfl_sync(0xFFFFFFFFu, v.b, r.from)}, o);
  } else {
    o[0] = x[1]; o[1] = x[0]; o[2] = x[3]; o[3] = x[2];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = (x[i] * r.c[i] + o[i] * r.s[i] + 8192) >> 14;
}
// Of 8-bit elements: both products in one instruction, of two 16-bit factors and two bytes.
template <int kLayout>
__device__ __forceinline__ void rotate(const Bytes& v, const Rotation<int8_t>& r, bool any, int (&x)[4]) {
  if (!any) return unpack(v, x);
  const uint32_t o = kLayout == kRotaryHalf ? __shfl_sync(0xFFFFFFFFu, v.w, r.from) : __byte_perm(v.w, 0, 0x2301);
  const int a = (int)__byte_perm(v.w, o, 0x5140), b = (int)__byte_perm(v.w, o, 0x7362);
  x[0] = __dp2a_lo(r.c[0], a, 8192) >> 14;
  x[1] = __dp2a_hi(r.c[1], a, 8192) >> 14;
  x[2] = __dp2a_lo(r.c[2], b, 8192) >> 14;
  x[3] = __dp2a_hi(r.c[3], b, 8192) >> 14;
}

// The smallest e with amax (8 + headroom) <= 1016 2^e; 11 at most, since headroom <= 8 and |x| <= 2^16: both of a pair's factors may be 1.
__device__ __forceinline__ int exponent(int amax, int headroom) {
  const int z = amax * (8 + headroom), e = max(22 - __clz(z), 0);      // z < 2^(e + 10)
  return e + (z > 1016 << e);
}

// The exponent of a lane's head. Of heads of less than a warp the largest of the lanes' exponents, each a bit in its head's 16 of a word: lanes
// with masks of their own would be reduced one head after another (the chunks above took 45 us, 41 with bits).
template <int D>
__device__ __forceinline__ int exponent(const int (&x)[4], int headroom, int lane) {
  const int m = max(max(abs(x[0]), abs(x[1])), max(abs(x[2]), abs(x[3])));
  if (D == 128) return exponent(__reduce_max_sync(0xFFFFFFFFu, m), headroom);
  const int field = D == 64 ? lane & 16 : 2 * (lane & 8);
  const unsigned mine = 1u << (exponent(m, headroom) + field);
  unsigned all;
  if (D == 64) {
    all = __reduce_or_sync(0xFFFFFFFFu, mine);
  } else {
    const unsigned low = __reduce_or_sync(0xFFFFFFFFu, lane < 16 ? mine : 0), high = __reduce_or_sync(0xFFFFFFFFu, lane < 16 ? 0 : mine);
    all = lane < 16 ? low : high;
  }
  return 31 - __clz((int)(all >> field & 0xFFFFu));
}

// The elements in 8 bits, -127 .. 127 (kFits: none is beyond 127 2^e).
template <bool kFits>
__device__ __forceinline__ uint32_t pack8(const int (&x)[4], int e) {
  const int half = (1 << e) >> 1;
  int y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = kFits ? (x[i] + half) >> e : max((x[i] + half) >> e, -127);
  uint32_t r;
  asm("{\n\t.reg .b32 t;\n\t"
      "cvt.pack.sat.s8.s32.b32 t, %4, %3, 0;\n\t"
      "cvt.pack.sat.s8.s32.b32 %0, %2, %1, t;\n\t}"
      : "=r"(r)
      : "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]));
  return r;
}

template <class X, int D, int kLayout, bool kVector>
__global__ void __launch_bounds__(32 * kAppendWarps, 6) append_kernel(const AttnArgs a, const CacheArgs c, const AppendArgs p, const int rows_log) {
  extern __shared__ uint8_t v8[];                  // [rows of the tile][kPitch]
  __shared__ int slots[4 * kAppendWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per_warp = 1 << rows_log, tile_log = rows_log + 3, tile = 1 << tile_log;
  const int row0 = blockIdx.x * tile, parts = gridDim.y, part = blockIdx.y;
  const int slot_end = c.blocks * kAttnBlock;      // below 2^31
  const int nq = a.heads * D, nk = a.kv * D, q_chunks = (nq + kChunk - 1) / kChunk;
  const int at = part * kChunk + lane * 4, h = at / D, d0 = at % D;          // the lane's keys and values
  const bool live = at < nk, rotary = a.rot != 0;
  const int q0 = part * q_chunks / parts, q1 = (part + 1) * q_chunks / parts;
  int first_row = -1, first_slot = -1, first_exps = 0;                       // the last first token of a block that was looked at: exponents of k, above four bits of v
  const int ahead = row0 + warp * per_warp + lane;                           // of the warp's rows, one to a lane
  const bool there = lane < per_warp && ahead < p.rows;
  const int slot_ahead = there ? p.slot[ahead] : -1, pos_ahead = there ? p.position[ahead] : 0;
  for (int i = 0; i < per_warp; ++i) {
    const int t = warp * per_warp + i, row = row0 + t;
    int slot = __shfl_sync(0xFFFFFFFFu, slot_ahead, i), pos = __shfl_sync(0xFFFFFFFFu, pos_ahead, i);
    if (row < p.rows) {
      const auto k4 = load<kVector>((const X*)p.k + row * p.ldk + at, live), v4 = load<kVector>((const X*)p.v + row * p.ldv + at, live);
      const bool bad = (rotary && (unsigned)pos >= (unsigned)a.positions) || slot < -1 || slot >= slot_end;
      if (bad && lane == 0 && part == 0) atomicAdd(a.status + 1, 1u);
      if (slot < 0 || slot >= slot_end) slot = -1;
      pos = min(max(pos, 0), a.positions - 1);
      const Rotation<X> rot = rotation<X, D, kLayout>(a, pos, lane);
      const X* from_q = (const X*)p.q + row * p.ldq + q0 * kChunk + lane * 4;
      int8_t* to_q = p.q8 + (long long)row * nq + q0 * kChunk + lane * 4;
      uint8_t* to_e = p.q_exp + (long long)row * a.heads + (q0 * kChunk + lane * 4) / D;
      int left = min(nq, q1 * kChunk) - q0 * kChunk - lane * 4;                // above 0: the lane has queries in this chunk
      auto q4 = load<kVector>(from_q, left > 0);
#pragma unroll 1
      for (int j = q0; j < q1; ++j, left -= kChunk, to_q += kChunk, to_e += kChunk / D) {
        int q[4];
        const auto now = q4;
        from_q += kChunk;
        q4 = load<kVector>(from_q, left > kChunk);
        rotate<kLayout>(now, rot, rotary, q);
        const int e = exponent<D>(q, 0, lane);
        if (left > 0) {
          *reinterpret_cast<uint32_t*>(to_q) = pack8<true>(q, e);
          if (lane * 4 % D == 0) *to_e = (uint8_t)e;
        }
      }
      if (slot >= 0) {
        const int off = slot % kAttnBlock, from = row - off, start = slot - off;
        const bool known = from == first_row && start == first_slot;           // another block's rows may lie as far behind the same row
        const long long head = (long long)(slot / kAttnBlock) * a.kv + h;
        int k[4], v[4], ek = 0, ev = 0;
        rotate<kLayout>(k4, rot, rotary, k);
        unpack(v4, v);
        if (off == 0) {
          ek = exponent<D>(k, a.k_headroom, lane);
          ev = exponent<D>(v, a.v_headroom, lane);
          if (live && d0 == 0) {
            c.k_exp[head] = (uint8_t)ek;
            c.v_exp[head] = (uint8_t)ev;
          }
        } else if (known || (from >= 0 && p.slot[from] == start)) {
          if (!known) {
            int x[4];
            unpack(load<kVector>((const X*)p.v + from * p.ldv + at, live), x);
            first_exps = exponent<D>(x, a.v_headroom, lane) << 4;
            rotate<kLayout>(load<kVector>((const X*)p.k + from * p.ldk + at, live),
                            rotation<X, D, kLayout>(a, min(max(p.position[from], 0), a.positions - 1), lane), rotary, x);
            first_exps |= exponent<D>(x, a.k_headroom, lane);
            first_row = from;
            first_slot = start;
          }
          ek = first_exps & 15;
          ev = first_exps >> 4;
        } else if (live) {
          ek = min((int)c.k_exp[head], kAttnMaxExp);
          ev = min((int)c.v_exp[head], kAttnMaxExp);
        }
        if (live) {
          *reinterpret_cast<uint32_t*>(c.k + (head * kAttnBlock + off) * D + d0) = pack8<false>(k, ek);
          *reinterpret_cast<uint32_t*>(v8 + t * kPitch + lane * 4) = pack8<false>(v, ev);
        }
      }
    }
    if (lane == 0) slots[t] = slot;
  }
  __syncthreads();
  // Values of neighbouring tokens of a dimension lie side by side: four to a word where their slots are.
  const int s0 = slots[0], elements = min(kChunk, nk - part * kChunk);
  const bool run = __syncthreads_and(s0 >= 0 && s0 % kAttnBlock + tile <= kAttnBlock && ((int)threadIdx.x >= tile || slots[threadIdx.x] == s0 + (int)threadIdx.x));
  if (run) {                                       // all rows of the tile one after another in one block
    int8_t* const base = c.v + ((long long)(s0 / kAttnBlock) * a.kv * D + part * kChunk) * kAttnBlock + s0 % kAttnBlock;
    const int shift = s0 & 3, words = tile / 4;      // of a dimension; the first and one more, behind them, may be partly of others
    auto store = [&](int el, int t) {
      const uint8_t* x = v8 + t * kPitch + el;
      int8_t* const to = base + el * kAttnBlock + t;
      if (t >= 0 && t + 4 <= tile) {
        *reinterpret_cast<uint32_t*>(to) = x[0] | x[kPitch] << 8 | x[2 * kPitch] << 16 | (uint32_t)x[3 * kPitch] << 24;
      } else {
        for (int j = max(0, -t); j < min(4, tile - t); ++j) to[j] = (int8_t)x[j * kPitch];
      }
    };
    for (int i = threadIdx.x; i < elements * words; i += 32 * kAppendWarps) store(i >> (tile_log - 2), (i & (words - 1)) * 4 - shift);
    if (shift)
      for (int el = threadIdx.x; el < elements; el += 32 * kAppendWarps) store(el, tile - shift);
    return;
  }
  for (int i = threadIdx.x; i < tile * elements; i += 32 * kAppendWarps) {
    const int t = i & (tile - 1), el = i >> tile_log, s = slots[t];
    if (s >= 0) c.v[((long long)(s / kAttnBlock) * a.kv * D + part * kChunk + el) * kAttnBlock + s % kAttnBlock] = (int8_t)v8[t * kPitch + el];
  }
}

template <class X, int D, int kLayout>
cudaError_t launch_append(const AttnArgs& a, const CacheArgs& c, const AppendArgs& p, cudaStream_t stream) {
  const int parts = (a.kv * D + kChunk - 1) / kChunk;
  // four rows to a warp where that still leaves two CTAs to an SM: their values make runs of 32 bytes (16384 rows of 32 bits: 136 us, 143 with two)
  const int rows_log = (long long)p.rows * parts >= 2ll * a.sms * (kAppendWarps << 2) ? 2 : 0, tile = kAppendWarps << rows_log;
  const dim3 grid((unsigned)((p.rows + tile - 1) / tile), (unsigned)parts);
  const size_t smem = (size_t)tile * kPitch;
  if (p.vector) append_kernel<X, D, kLayout, true><<<grid, 32 * kAppendWarps, smem, stream>>>(a, c, p, rows_log);
  else append_kernel<X, D, kLayout, false><<<grid, 32 * kAppendWarps, smem, stream>>>(a, c, p, rows_log);
  return cudaGetLastError();
}

template <class X, int kLayout>
cudaError_t launch_append(const AttnArgs& a, const CacheArgs& c, const AppendArgs& p, cudaStream_t stream) {
  return a.dim == 128 ? launch_append<X, 128, kLayout>(a, c, p, stream)
                      : a.dim == 64 ? launch_append<X, 64, kLayout>(a, c, p, stream) : launch_append<X, 32, kLayout>(a, c, p, stream);
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
