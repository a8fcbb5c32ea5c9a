// Attention of many rows (include/iodf.h: iodf_attn_forward): prompts, chunks of them, images.
//
// A unit of work is 128 rows of a request and the keys of one head of the cache; rows are (token, query head of the group) pairs, so that
// all query heads of a group share the keys and values that are read. The rows are the MMA's M: a thread of the softmax owns a row.
//   pass 1: S = Q K^T per block of 128 keys, the largest t of each row
//   pass 2: S again, weights p = 256 hi + lo (8 unsigned and 8 signed bits), O_hi += hi V, O_lo += lo V in tensor memory
// With the maximum known no sum is ever rescaled. Two groups of four warps take the blocks in turn; S, and the weights in shared
// memory, exist twice, so that one group computes while the other's MMAs run.
// What bounds it: about ten integer instructions per score on the softmax warps (64 a clock and SM for most of them).
#include <algorithm>

#include "../../include/iodf.h"
#include "attn_device.cuh"
#include "attn_kernels.h"
#include "iodf_dev.h"
#include "ptx_attn.cuh"

namespace iodf {
namespace {

constexpr int kRows = 128;
constexpr int kThreads2 = 384;           // warp 0 copies, 1 MMAs, 2-3 queries, 4-7 and 8-11 softmax
constexpr int kKRing = 3, kVRing = 2, kUnits = 4, kMeta = 8;
constexpr int kBlockBytes = 16384;       // of a ring's slot: 128 rows of up to 128 bytes
constexpr int kTableBytes = kWeightSegments * 128;                 // a copy of the table for each lane: no bank is asked twice
constexpr int kSmem = kTableBytes + (2 + kKRing + kVRing + 4) * kBlockBytes;

struct Unit {
  int request, head, row0, len;          // rows of the request: [row0, row0 + len)
  int tile, held;
  int b0, b1;                            // blocks that its rows see
};

struct Shared {
  uint64_t kfull[kKRing], kempty[kKRing], vfull[kVRing], vempty[kVRing], qfull[2], qempty[2], sfull[2], sempty[2], pfull[2], pempty[2];
  uint64_t ofull, oempty, ufull[kUnits], uempty[kUnits];
  uint32_t abort_flag, tmem;
  Unit units[kUnits];
  int2 meta[kMeta];                      // exponents of a block's keys and values, -1: nobody sees it
  int top[2][kRows], vexp[2][kRows];     // of the two groups
  long long sum[2][kRows];
};

struct Ring {                            // slot and phase, counted
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int size) {
    if (++slot == size) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

struct Tile {                            // what every role derives from a unit
  int flat0, flats;                      // rows (token, head) of the unit: [flat0, flats)
  __device__ __forceinline__ Tile(const AttnArgs& a, const Unit& u) : flat0(u.tile * kRows), flats(min(u.len * a.group, (u.tile + 1) * kRows)) {}
  __device__ __forceinline__ int position(const AttnArgs& a, const Unit& u, int flat) const { return u.held - u.len + flat / a.group; }
};

// Finds the units of a CTA, one after another: requests 32 at a time over the lanes of a warp.
struct Finder {
  int base = 0, before = 0;              // first request of the 32; units before them
  int start = 0, len = 0, tiles = 0;     // of the lane's request
  int upto = 0, all = 0;                 // inclusive sum of units over the lanes, and over all of them
  bool loaded = false;
  __device__ __forceinline__ void load(const AttnArgs& a, const ForwardArgs& f, int lane) {
    const int q = base + lane;
    int s0 = 0, s1 = 0;
    if (q < f.n) {
      s0 = f.row_start[q];
      s1 = f.row_start[q + 1];
    }
    start = min(max(s0, 0), f.rows);
    len = max(min(max(s1, 0), f.rows) - start, 0);
    tiles = (len * a.group + kRows - 1) / kRows;
    upto = tiles * a.kv;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int o = __shfl_up_sync(0xFFFFFFFFu, upto, d);
      if (lane >= d) upto += o;
    }
    all = __shfl_sync(0xFFFFFFFFu, upto, 31);
    loaded = true;
  }
  __device__ __forceinline__ bool find(const AttnArgs& a, const ForwardArgs& f, int unit, int lane, Unit* u) {
    if (!loaded) load(a, f, lane);
    while (unit >= before + all) {
      before += all;
      base += 32;
      if (base >= f.n) return false;
      load(a, f, lane);
    }
    const int from = __ffs((int)__ballot_sync(0xFFFFFFFFu, unit < before + upto)) - 1;
    const int in = unit - before - (__shfl_sync(0xFFFFFFFFu, upto, from) - __shfl_sync(0xFFFFFFFFu, tiles, from) * a.kv);
    u->request = base + from;
    u->row0 = __shfl_sync(0xFFFFFFFFu, start, from);
    u->len = __shfl_sync(0xFFFFFFFFu, len, from);
    u->tile = __shfl_sync(0xFFFFFFFFu, tiles, from) - 1 - in / a.kv;       // the last rows, which see the most keys, first
    u->head = in % a.kv;
    u->held = min(max(f.held[u->request], 0), f.width * kAttnBlock);
    const Tile t(a, *u);
    const Range low = visible(a, t.position(a, *u, t.flat0), u->held), high = visible(a, t.position(a, *u, t.flats - 1), u->held);
    u->b0 = low.first / kAttnBlock;
    u->b1 = high.last <= low.first ? u->b0 : (high.last + kAttnBlock - 1) / kAttnBlock;
    return true;
  }
};

// Weights of four scores, as the bytes hi and lo of p + 128 (lo with its highest bit turned over is signed).
__device__ __forceinline__ void split4(const uint32_t (&w)[4], uint32_t* hi, uint32_t* lo) {
  const uint32_t a = __byte_perm(w[0], w[1], 0x5140), b = __byte_perm(w[2], w[3], 0x5140);    // lo lo hi hi
  *lo = __byte_perm(a, b, 0x5410) ^ 0x80808080u;
  *hi = __byte_perm(a, b, 0x7632);
}

template <int D>
__global__ void __launch_bounds__(kThreads2, 1) tile_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                                                            const AttnArgs a, const CacheArgs c, const ForwardArgs f) {
  extern __shared__ uint8_t raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 8191) & ~(uintptr_t)8191);
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t table = ptx::smem_u32(smem), qbuf = table + kTableBytes, kbuf = qbuf + 2 * kBlockBytes, vbuf = kbuf + kKRing * kBlockBytes,
                 pbuf = vbuf + kVRing * kBlockBytes;
  volatile uint32_t* const abort_flag = &sh.abort_flag;
  if (tid == 0) {
    auto init = [](uint64_t* bars, int n, int count) {
      for (int i = 0; i < n; ++i) ptx::mbar_init(ptx::smem_u32(bars + i), count);
    };
    init(sh.kfull, kKRing, 1);
    init(sh.kempty, kKRing, 1);
    init(sh.vfull, kVRing, 1);
    init(sh.vempty, kVRing, 1);
    init(sh.qfull, 2, 2);
    init(sh.qempty, 2, 1);
    init(sh.sfull, 2, 2);
    init(sh.sempty, 2, 4);
    init(sh.pfull, 2, 4);
    init(sh.pempty, 2, 1);
    init(&sh.ofull, 1, 1);
    init(&sh.oempty, 1, 8);
    init(sh.ufull, kUnits, 1);
    init(sh.uempty, kUnits, 11);
    ptx::mbar_init_fence();
    sh.abort_flag = 0;
  }
  for (int i = tid; i < kWeightSegments * 32; i += kThreads2) reinterpret_cast<int*>(smem)[i] = weight_word(i / 32);
  if (warp == 2) ptx::tmem_alloc(ptx::smem_u32(&sh.tmem), 512);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = sh.tmem, o_hi = tmem + 256, o_lo = o_hi + D;
  auto wait = [&](uint64_t* bar, uint32_t phase) { return ptx::quick_wait(abort_flag, a.status, bar, phase, kSpinLimit); };
  auto warp_wait = [&](uint64_t* bar, uint32_t phase) { return __all_sync(0xFFFFFFFFu, wait(bar, phase)) != 0; };   // all lanes go on, or none
  // the unit of a consumer's turn; false when there are no more
  auto take = [&](const Ring& r, Unit* u) {
    if (!wait(&sh.ufull[r.slot], r.phase)) return false;
    *u = sh.units[r.slot];
    return u->request >= 0;
  };

  if (warp == 0) {
    // Copies, and everything that is read to find out what to copy: units, blocks and their exponents, 32 over the lanes.
    Finder finder;
    Ring kr, vr, ur;
    int count = 0;                                      // blocks, for meta
    bool ok = true;
    for (int round = 0; ok; ++round, ur.next(kUnits)) {
      const int unit = round * (int)gridDim.x + ((round & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
      Unit u;
      const bool more = finder.find(a, f, unit, lane, &u);
      if (!more) u.request = -1;
      ok = warp_wait(&sh.uempty[ur.slot], ur.phase ^ 1);
      if (!ok) break;
      if (lane == 0) {
        sh.units[ur.slot] = u;
        ptx::mbar_arrive(ptx::smem_u32(&sh.ufull[ur.slot]));
        if (more && u.tile == 0 && u.head == 0 && f.held[u.request] != u.held) atomicAdd(a.status + 1, 1u);
      }
      if (!more) break;
      for (int pass = 0; pass < 2 && ok; ++pass) {
        int id = 0, ek = 0, ev = 0;
        for (int b = u.b0; b < u.b1 && ok; ++b, ++count) {
          const int in = (b - u.b0) & 31;
          if (in == 0) {
            id = b + lane < u.b1 ? f.table[(long long)u.request * f.ldt + b + lane] : 0;
            const bool good = (unsigned)id < (unsigned)c.blocks;
            if (!good && pass) atomicAdd(a.status + 1, 1u);
            if (!good) id = 0;
            const long long at = (long long)id * a.kv + u.head;
            ek = min((int)c.k_exp[at], kAttnMaxExp);
            ev = good ? min((int)c.v_exp[at], kAttnMaxExp) : -1;
          }
          const int at = __shfl_sync(0xFFFFFFFFu, id, in) * a.kv + u.head;
          const int2 m = make_int2(__shfl_sync(0xFFFFFFFFu, ek, in), __shfl_sync(0xFFFFFFFFu, ev, in));
          ok = warp_wait(&sh.kempty[kr.slot], kr.phase ^ 1);
          if (ok && ptx::elect_one()) {
            sh.meta[count % kMeta] = m;
            const uint32_t bar = ptx::smem_u32(&sh.kfull[kr.slot]);
            ptx::mbar_expect_tx(bar, kAttnBlock * D);
            ptx::tile_g2s(kbuf + kr.slot * kBlockBytes, &kmap, 0, at * kAttnBlock, bar);
          }
          __syncwarp();
          kr.next(kKRing);
          if (pass && ok) {
            ok = warp_wait(&sh.vempty[vr.slot], vr.phase ^ 1);
            if (ok && ptx::elect_one()) {
              const uint32_t bar = ptx::smem_u32(&sh.vfull[vr.slot]);
              ptx::mbar_expect_tx(bar, kAttnBlock * D);
              ptx::tile_g2s(vbuf + vr.slot * kBlockBytes, &vmap, 0, at * D, bar);
            }
            __syncwarp();
            vr.next(kVRing);
          }
        }
      }
    }
    // whoever fills a ring waits until the MMAs have given all of it back: no copy or arrival outlives the CTA
    for (int i = 0; ok && i < kKRing; ++i, kr.next(kKRing)) ok = wait(&sh.kempty[kr.slot], kr.phase ^ 1);
    for (int i = 0; ok && i < kVRing; ++i, vr.next(kVRing)) ok = wait(&sh.vempty[vr.slot], vr.phase ^ 1);
  } else if (warp == 1) {
    if (ptx::elect_one()) {
      constexpr uint32_t id_s = idesc_i8(kRows, kAttnBlock, false, false), id_hi = idesc_i8(kRows, D, true, false), id_lo = idesc_i8(kRows, D, false, false);
      constexpr uint32_t hi_d = rows_hi(D), hi_128 = rows_hi(128);
      Ring kr, vr, ur, qr, sr, orr;                     // sr: S and its barriers, two in turn
      uint32_t pphases = 0;                             // of the two groups' weights
      Unit u;
      bool ok = true;
      auto scores = [&](uint32_t q) {                   // S of the next block
        ok = ok && wait(&sh.kfull[kr.slot], kr.phase) && wait(&sh.sempty[sr.slot], sr.phase ^ 1);
        if (!ok) return;
        ptx::tc_fence_after();
        const uint32_t k = rows_lo(kbuf + kr.slot * kBlockBytes);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) ptx::umma_i8_hl(tmem + sr.slot * 128, q + 2 * i, hi_d, k + 2 * i, hi_d, id_s, i > 0);
        ptx::umma_commit(ptx::smem_u32(&sh.kempty[kr.slot]));
        ptx::umma_commit(ptx::smem_u32(&sh.sfull[sr.slot]));
        ptx::mbar_arrive(ptx::smem_u32(&sh.sfull[sr.slot]));      // what the copying warp wrote of the block is passed on
        kr.next(kKRing);
        sr.next(2);
      };
      for (; ok && take(ur, &u); ur.next(kUnits)) {
        const int n = u.b1 - u.b0;
        ok = wait(&sh.qfull[qr.slot], qr.phase);
        ptx::tc_fence_after();
        const uint32_t q = rows_lo(qbuf + qr.slot * kBlockBytes);
        for (int j = 0; j < n && ok; ++j) scores(q);
        int ps = sr.slot;                               // the weights of a block are where its S is
        for (int j = 0; j < n + 2 && ok; ++j) {
          if (j >= 2) {
            if (j == 2) ok = wait(&sh.oempty, orr.phase ^ 1);
            ok = ok && wait(&sh.pfull[ps], (pphases >> ps) & 1) && wait(&sh.vfull[vr.slot], vr.phase);
            if (!ok) break;
            ptx::tc_fence_after();
            const uint32_t p = rows_lo(pbuf + ps * 2 * kBlockBytes), v = rows_lo(vbuf + vr.slot * kBlockBytes);
#pragma unroll
            for (int i = 0; i < 4; ++i) ptx::umma_i8_hl(o_hi, p + 2 * i, hi_128, v + 2 * i, hi_128, id_hi, j > 2 || i > 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) ptx::umma_i8_hl(o_lo, p + (kBlockBytes >> 4) + 2 * i, hi_128, v + 2 * i, hi_128, id_lo, j > 2 || i > 0);
            ptx::umma_commit(ptx::smem_u32(&sh.vempty[vr.slot]));
            ptx::umma_commit(ptx::smem_u32(&sh.pempty[ps]));
            vr.next(kVRing);
            pphases ^= 1u << ps;
            ps ^= 1;
          }
          if (j < n) scores(q);
        }
        if (ok && n) {
          ptx::umma_commit(ptx::smem_u32(&sh.ofull));
          orr.next(1);
        }
        // all MMAs that read the queries are committed before this arrival comes
        if (ok) ptx::umma_commit(ptx::smem_u32(&sh.qempty[qr.slot]));
        qr.next(2);
        ptx::mbar_arrive(ptx::smem_u32(&sh.uempty[ur.slot]));
      }
      // no arrival of a commit is left to come when the CTA leaves: of S and O the softmax warps wait for all, of the rings their fillers
      for (int i = 0; ok && i < 2; ++i) ok = wait(&sh.pempty[i], ((pphases >> i) & 1) ^ 1);
    }
    __syncwarp();
  } else if (warp < 4) {
    // Queries: rows of D bytes into the layout of the MMA's operand.
    const int t = tid - 64;
    Ring qr, ur;
    Unit u;
    bool ok = true;
    for (; ok && __all_sync(0xFFFFFFFFu, take(ur, &u)); ur.next(kUnits), qr.next(2)) {
      ok = warp_wait(&sh.qempty[qr.slot], qr.phase ^ 1);
      const Tile tile(a, u);
      for (int i = t; ok && i < kRows * (D / 16); i += 64) {
        const int r = i / (D / 16), piece = i % (D / 16), flat = tile.flat0 + r;
        if (flat < tile.flats) {
          const long long row = u.row0 + flat / a.group;
          const int4 v = *reinterpret_cast<const int4*>(f.q8 + (row * a.heads + u.head * a.group + flat % a.group) * D + piece * 16);
          ptx::sts128(qbuf + qr.slot * kBlockBytes + swizzled(r, piece, D), v.x, v.y, v.z, v.w);
        }
      }
      ptx::fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        ptx::mbar_arrive(ptx::smem_u32(&sh.qfull[qr.slot]));
        ptx::mbar_arrive(ptx::smem_u32(&sh.uempty[ur.slot]));
      }
    }
    for (int i = 0; ok && i < 2; ++i, qr.next(2)) ok = wait(&sh.qempty[qr.slot], qr.phase ^ 1);
  } else {
    const int w = (warp - 4) >> 2, quarter = warp & 3, r = quarter * 32 + lane;          // group, lanes of tensor memory, row of the tile
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16, s_mem = tmem + lanes + w * 128, words = table + lane * 4;
    const uint32_t p_hi = pbuf + w * 2 * kBlockBytes, p_lo = p_hi + kBlockBytes;
    Ring ur, orr;
    uint32_t sphase = 0, pphase = 1;
    int count = 0;                                      // blocks of the units before
    Unit u;
    bool ok = true;
    while (ptx::all_agree(1, 256, take(ur, &u))) {      // in step: there are barriers below, whatever the other waits return
      const Tile tile(a, u);
      const int flat = tile.flat0 + r, n = u.b1 - u.b0;
      const bool live = flat < tile.flats;
      const long long row = u.row0 + (live ? flat : tile.flat0) / a.group;
      const int head = u.head * a.group + flat % a.group;
      const Range see = visible(a, tile.position(a, u, live ? flat : tile.flat0), u.held);
      const int eq = live ? min((int)f.q_exp[row * a.heads + head], kAttnMaxExp) : 0;
      // blocks in [whole0, whole1) are seen whole by every row
      const Range low = visible(a, tile.position(a, u, tile.flat0), u.held), high = visible(a, tile.position(a, u, tile.flats - 1), u.held);
      const int whole0 = (high.first + kAttnBlock - 1) / kAttnBlock, whole1 = max(low.last, 0) / kAttnBlock;
      int T = INT32_MIN, V = 0;
      // S and weights alternate between the groups over all blocks of all units, so who begins depends on the blocks before
      // (each pass has n of them)
      for (int j = (w ^ count) & 1; j < n; j += 2) {
        ok = ok && warp_wait(&sh.sfull[w], sphase);
        sphase ^= 1;
        if (!ok) break;
        ptx::tc_fence_after();
        const int b = u.b0 + j;
        const int2 m = sh.meta[(count + j) % kMeta];
        const bool whole = b >= whole0 && b < whole1;
        int top = INT32_MIN;
#pragma unroll
        for (int c0 = 0; c0 < kAttnBlock; c0 += 32) {
          uint32_t s[32];
          ptx::tmem_ld32(s_mem + c0, s);
          ptx::tmem_ld_wait32(s);
          if (whole) {
#pragma unroll
            for (int i = 0; i < 32; ++i) top = max(top, (int)s[i]);
          } else {
            const int first = see.first - b * kAttnBlock - c0, last = see.last - b * kAttnBlock - c0;
#pragma unroll
            for (int i = 0; i < 32; ++i) top = i >= first && i < last ? max(top, (int)s[i]) : top;
          }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.sempty[w]));
        if (m.y >= 0 && top != INT32_MIN) {
          T = max(T, score_octaves(top, score_multiplier(a.score_m0, eq + m.x, a.score_s)));
          V = max(V, m.y);
        }
      }
      count += n;
      sh.top[w][r] = T;
      sh.vexp[w][r] = V;
      ptx::named_barrier(1, 256);
      T = max(T, sh.top[w ^ 1][r]);
      V = max(V, sh.vexp[w ^ 1][r]);
      long long L = 0;
      for (int j = (w ^ count) & 1; j < n; j += 2) {
        ok = ok && warp_wait(&sh.sfull[w], sphase) && warp_wait(&sh.pempty[w], pphase);
        sphase ^= 1;
        pphase ^= 1;
        if (!ok) break;
        ptx::tc_fence_after();
        const int b = u.b0 + j;
        const int2 m = sh.meta[(count + j) % kMeta];
        const bool whole = b >= whole0 && b < whole1 && m.y >= 0;
        const int W = score_multiplier(a.score_m0, eq + m.x, a.score_s), d = max(V - m.y, 0), C = -(T + 8192 * d);
        const int first = m.y < 0 ? INT32_MAX : see.first - b * kAttnBlock, last = see.last - b * kAttnBlock;
        uint32_t sum = 0;
#pragma unroll
        for (int c0 = 0; c0 < kAttnBlock; c0 += 32) {
          uint32_t s[32];
          ptx::tmem_ld32(s_mem + c0, s);
          ptx::tmem_ld_wait32(s);
          uint32_t hi[8], lo[8];
          auto weights = [&](auto masked) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              uint32_t x[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                int t = max(score_octaves((int)s[i + e], W) + C, kWeightLow);
                if (masked.value) t = c0 + i + e >= first && c0 + i + e < last ? t : kWeightLow;
                x[e] = weight_bits(t, (int)ptx::lds32((uint32_t)(t & ((kWeightSegments - 1) << 7)) | words));
                sum += x[e];
              }
              split4(x, &hi[i / 4], &lo[i / 4]);
            }
          };
          if (whole) weights(std::false_type());
          else weights(std::true_type());
          const int piece = c0 / 16;
          ptx::sts128(p_hi + swizzled(r, piece, 128), hi[0], hi[1], hi[2], hi[3]);
          ptx::sts128(p_hi + swizzled(r, piece + 1, 128), hi[4], hi[5], hi[6], hi[7]);
          ptx::sts128(p_lo + swizzled(r, piece, 128), lo[0], lo[1], lo[2], lo[3]);
          ptx::sts128(p_lo + swizzled(r, piece + 1, 128), lo[4], lo[5], lo[6], lo[7]);
        }
        ptx::tc_fence_before();
        ptx::fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive(ptx::smem_u32(&sh.sempty[w]));
          ptx::mbar_arrive(ptx::smem_u32(&sh.pfull[w]));
        }
        L += (long long)(sum - kAttnBlock * kWeightBias) << d;
      }
      count += n;
      sh.sum[w][r] = L;
      ptx::named_barrier(1, 256);
      L += sh.sum[w ^ 1][r];
      if (n) {
        ok = ok && warp_wait(&sh.ofull, orr.phase);
        orr.next(1);
        ptx::tc_fence_after();
      }
      const Reciprocal rec = reciprocal(max(L, 1ll), V);
      const long long y_at = row * f.ldy + head * D;
#pragma unroll 1
      for (int c0 = w * (D / 2); c0 < (w + 1) * (D / 2); c0 += 16) {
        uint32_t h[16], l[16];
        if (n) {
          ptx::tmem_ld16(o_hi + lanes + c0, h);
          ptx::tmem_ld16(o_lo + lanes + c0, l);
          ptx::tmem_ld_wait16(h);
          ptx::tmem_ld_wait16_nosync(l);
        }
        int y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const long long A = ((long long)(int)h[i] << 8) + (int)l[i];
          y[i] = requantised(L ? quotient(A, rec) : 0, a.out[head * D + c0 + i], a.lo, a.hi);
        }
        if (live && ok) {
          if (a.y_bytes == 1) {
            int8_t* p = (int8_t*)f.y + y_at + c0;
            uint32_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              v[i] = (uint32_t)(y[4 * i] & 255) | (uint32_t)(y[4 * i + 1] & 255) << 8 | (uint32_t)(y[4 * i + 2] & 255) << 16 | (uint32_t)y[4 * i + 3] << 24;
            if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) {
              *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) p[i] = (int8_t)y[i];
            }
          } else {
            int* p = (int*)f.y + y_at + c0;
            if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
              for (int i = 0; i < 16; i += 4) *reinterpret_cast<int4*>(p + i) = make_int4(y[i], y[i + 1], y[i + 2], y[i + 3]);
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) p[i] = y[i];
            }
          }
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (n) ptx::mbar_arrive(ptx::smem_u32(&sh.oempty));
        ptx::mbar_arrive(ptx::smem_u32(&sh.uempty[ur.slot]));
      }
      ur.next(kUnits);
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (warp == 2) ptx::tmem_dealloc(tmem, 512);
}

}  // namespace

cudaError_t configure_attn_tile() {
  const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaFuncSetAttribute(tile_kernel<32>, attr, kSmem + 8192);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(tile_kernel<64>, attr, kSmem + 8192);
  return e == cudaSuccess ? cudaFuncSetAttribute(tile_kernel<128>, attr, kSmem + 8192) : e;
}

cudaError_t launch_attn_tile(const AttnArgs& a, const CacheArgs& c, const ForwardArgs& f, const CUtensorMap& k_map, const CUtensorMap& v_map,
                             cudaStream_t stream) {
  const long long units = ((long long)f.rows * a.group / kRows + f.n) * a.kv;             // at most
  const int grid = (int)std::min<long long>(a.sms, units);
  const auto kernel = a.dim == 128 ? tile_kernel<128> : a.dim == 64 ? tile_kernel<64> : tile_kernel<32>;
  kernel<<<grid, kThreads2, kSmem + 8192, stream>>>(k_map, v_map, a, c, f);
  return cudaGetLastError();
}

}  // namespace iodf
