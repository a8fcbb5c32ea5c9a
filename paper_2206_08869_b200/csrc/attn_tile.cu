// Attention of many rows (include/iodf.h: iodf_attn_forward): prompts, chunks of them, images.
//
// A unit of work is 128 rows of a request and the keys of one head of the cache; rows are (token, query head of the group) pairs, so that
// all query heads of a group share the keys and values that are read. The rows are the MMA's M: a thread of the softmax owns a row.
//   pass 1: S = Q K^T per block of 128 keys, the largest t of each row
//   pass 2: S again, weights p = 256 hi + lo (8 unsigned and 8 signed bits), O_hi += hi V, O_lo += lo V in tensor memory
// With the maximum known no sum is ever rescaled. Two groups of four warps take the blocks in turn; S, and the weights in shared
// memory, exist twice, so that one group computes while the other's MMAs run.
// What bounds it: the integer instructions of a weight (a product's high word at a quarter of the usual rate, a clip, a table word, a float
// add, the split into bytes), 14 clocks for 128 scores and a quarter of an SM alone and 18 to 21 beside MMAs that read shared memory,
// through which the table's words and the weights go too: 2300 to 2700 clocks for a block of 128 x 128, where its MMAs take 1400 with
// D = 128. A product of doubles for the high word, or a polynomial for the table's word, cost as much or more.
// 16384 tokens of a prompt, 32 heads of 128 over 8, causal: 3.32 ms (8 softmax warps 4.16, 16 3.68; copies in the order of the MMAs and the
// unit's outputs beside the next one's first pass 3.46; waits that the hardware suspends 3.32). 128 images of 256 tokens, 4 heads of 64: 58.5 us,
// where a unit of two blocks has twice its instructions' time in waits of one step for the other.
#include <algorithm>

#include "../../include/iodf.h"
#include "attn_device.cuh"
#include "attn_kernels.h"
#include "iodf_dev.h"
#include "ptx_attn.cuh"

namespace iodf {
namespace {

constexpr int kRows = 128, kHalf = kAttnBlock / 2;
constexpr int kSoft = 16;                // softmax warps: two groups that take blocks in turn, two halves of a block's keys, 32 rows each
constexpr int kThreads2 = 128 + 32 * kSoft;                       // warp 0 copies, 1 MMAs, 2 units, 3 queries, then softmax
constexpr int kRing = 5, kUnits = 3;     // stages, units
constexpr int kScores = 6;               // barriers of S: see `place`
constexpr int kBlockBytes = 16384;       // of a ring's slot: 128 rows of up to 128 bytes
constexpr int kTableBytes = kWeightSegments * 128;                 // a copy of the table for each lane: no bank is asked twice
constexpr int kSmem = kTableBytes + (2 + kRing + 4) * kBlockBytes;
// Blocks at the first pass's start that the second group takes alone while the first one stores the unit before (4 or 16: 2 % slower).
constexpr int kLead = 8;

struct Unit {
  int request, head, row0, len;          // rows of the request: [row0, row0 + len)
  int tile, held;
  int b0, b1;                            // blocks that its rows see
};

struct Shared {
  uint64_t full[kRing], empty[kRing], qfull[2], qempty[2], sfull[kScores], sempty[kScores], pfull[2], pempty[2];
  uint64_t ofull, oempty, ufull[kUnits], uempty[kUnits];
  uint32_t abort_flag, tmem;
  Unit units[kUnits];
  int ids[kUnits][kAttnMaxBlocks];       // blocks of the unit; -1: outside the cache, nobody sees it
  uint16_t exps[kUnits][kAttnMaxBlocks]; // their exponents: of the keys, above eight bits of the values, kBad
  int multipliers[2 * kAttnMaxExp + 1];  // W by the sum of the exponents
  int top[4][kRows], vexp[4][kRows];     // of the groups' halves
  long long sum[4][kRows];
};

constexpr int kBad = 1 << 15;

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
    const int mine = __shfl_sync(0xFFFFFFFFu, tiles, from) * a.kv, in = unit - before - (__shfl_sync(0xFFFFFFFFu, upto, from) - mine);
    if ((unsigned)in >= (unsigned)mine) return false;                        // requests that share rows, more of them than can be counted
    u->request = base + from;
    u->row0 = __shfl_sync(0xFFFFFFFFu, start, from);
    u->len = __shfl_sync(0xFFFFFFFFu, len, from);
    u->tile = mine / a.kv - 1 - in / a.kv;       // the last rows, which see the most keys, first
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

// Four outputs of a word, saturated to signed 8 bits.
__device__ __forceinline__ uint32_t packed(int a, int b, int c, int d) {
  uint32_t r;
  asm("{\n\t.reg .b32 t;\n\t"
      "cvt.pack.sat.s8.s32.b32 t, %4, %3, 0;\n\t"
      "cvt.pack.sat.s8.s32.b32 %0, %2, %1, t;\n\t}"
      : "=r"(r)
      : "r"(a), "r"(b), "r"(c), "r"(d));
  return r;
}

template <int D>
__global__ void __launch_bounds__(kThreads2, 1) tile_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                                                            const AttnArgs a, const CacheArgs c, const ForwardArgs f) {
  extern __shared__ uint8_t raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 8191) & ~(uintptr_t)8191);
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t table = ptx::smem_u32(smem), qbuf = table + kTableBytes, ring = qbuf + 2 * kBlockBytes, pbuf = ring + kRing * kBlockBytes;
  volatile uint32_t* const abort_flag = &sh.abort_flag;
  if (tid == 0) {
    auto init = [](uint64_t* bars, int n, int count) {
      for (int i = 0; i < n; ++i) ptx::mbar_init(ptx::smem_u32(bars + i), count);
    };
    init(sh.full, kRing, 1);
    init(sh.empty, kRing, 1);
    init(sh.qfull, 2, 1);
    init(sh.qempty, 2, 1);
    init(sh.sfull, kScores, 1);
    init(sh.sempty, kScores, kSoft / 2);
    init(sh.pfull, 2, kSoft / 2);
    init(sh.pempty, 2, 1);
    init(&sh.ofull, 1, 1);
    init(&sh.oempty, 1, kSoft / 2);
    init(sh.ufull, kUnits, 1);
    init(sh.uempty, kUnits, 3 + kSoft);
    ptx::mbar_init_fence();
    sh.abort_flag = 0;
  }
  for (int i = tid; i < kWeightSegments * 32; i += kThreads2) reinterpret_cast<int*>(smem)[i] = weight_word(i / 32);
  if (tid <= 2 * kAttnMaxExp) sh.multipliers[tid] = score_multiplier(a.score_m0, tid, a.score_s);
  if (warp == 2) ptx::tmem_alloc(ptx::smem_u32(&sh.tmem), 512);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = sh.tmem, o_hi = tmem + 256, o_lo = o_hi + D;
  auto wait = [&](uint64_t* bar, uint32_t phase) { return ptx::quick_wait(abort_flag, a.status, bar, phase, kSpinLimit); };
  auto warp_wait = [&](uint64_t* bar, uint32_t phase) { return __all_sync(0xFFFFFFFFu, wait(bar, phase)) != 0; };   // all lanes go on, or none
  // S of a block in the first pass: 0 to 3, each read by half of a group; of the lead 4 and 5, which lie where 0 and 1 do but have barriers of
  // their own: their reader is another one than that of 0, and who waits for a phase must not be two phases late. In the second pass
  // the groups alternate, in S 0 and 1. S 2 and 3 lie where O will be.
  auto place = [](int j) { return j < kLead ? 4 + (j & 1) : j & 3; };
  // the unit of a consumer's turn; false when there are no more
  auto take = [&](const Ring& r, Unit* u) {
    if (!wait(&sh.ufull[r.slot], r.phase)) return false;
    *u = sh.units[r.slot];
    return u->request >= 0;
  };

  if (warp == 0) {
    if (ptx::elect_one()) {
      Ring r, ur;
      Unit u;
      bool ok = true;
      auto copy = [&](const CUtensorMap* map, int row) {
        ok = ok && wait(&sh.empty[r.slot], r.phase ^ 1);
        if (!ok) return;
        const uint32_t bar = ptx::smem_u32(&sh.full[r.slot]);
        ptx::mbar_expect_tx(bar, kAttnBlock * D);
        ptx::tile_g2s(ring + r.slot * kBlockBytes, map, 0, row, bar);
        r.next(kRing);
      };
      for (; ok && take(ur, &u); ur.next(kUnits)) {    // in the order in which the MMAs read them
        const int* ids = sh.ids[ur.slot];
        const int n = u.b1 - u.b0;
        auto at = [&](int j) { return max(ids[j], 0) * a.kv + u.head; };
        for (int j = 0; j < n && ok; ++j) copy(&kmap, at(j) * kAttnBlock);
        for (int j = -2; j < n && ok; ++j) {
          if (j + 2 < n) copy(&kmap, at(j + 2) * kAttnBlock);
          if (j >= 0) copy(&vmap, at(j) * D);
        }
        ptx::mbar_arrive(ptx::smem_u32(&sh.uempty[ur.slot]));
      }
      // whoever fills a ring waits until the MMAs have given all of it back: no copy or arrival outlives the CTA
      for (int i = 0; ok && i < kRing; ++i, r.next(kRing)) ok = wait(&sh.empty[r.slot], r.phase ^ 1);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (ptx::elect_one()) {
      constexpr uint32_t id_s = idesc_i8(kRows, kAttnBlock, false, false), id_hi = idesc_i8(kRows, D, true, false), id_lo = idesc_i8(kRows, D, false, false);
      constexpr uint32_t hi_d = rows_hi(D), hi_128 = rows_hi(128);
      Ring r, ur, qr, orr;
      uint32_t pphases = 0, sphases = 0;                // of each group's weights and of each S, in bits
      Unit u;
      bool ok = true;
      auto scores = [&](uint32_t q, int slot) {         // S of the next block
        ok = ok && wait(&sh.full[r.slot], r.phase) && wait(&sh.sempty[slot], (sphases >> slot & 1) ^ 1);
        if (!ok) return;
        ptx::tc_fence_after();
        const uint32_t k = rows_lo(ring + r.slot * kBlockBytes);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) ptx::umma_i8_hl(tmem + (slot & 3) * 128, q + 2 * i, hi_d, k + 2 * i, hi_d, id_s, i > 0);
        ptx::umma_commit(ptx::smem_u32(&sh.empty[r.slot]));
        ptx::umma_commit(ptx::smem_u32(&sh.sfull[slot]));
        r.next(kRing);
        sphases ^= 1u << slot;
      };
      for (; ok && take(ur, &u); ur.next(kUnits)) {
        const int n = u.b1 - u.b0;
        bool o_free = false;                            // the unit before has been read out of O
        auto free_o = [&] {
          if (!o_free) ok = ok && wait(&sh.oempty, orr.phase ^ 1);
          o_free = true;
        };
        ok = wait(&sh.qfull[qr.slot], qr.phase);
        ptx::tc_fence_after();
        const uint32_t q = rows_lo(qbuf + qr.slot * kBlockBytes);
        auto free_s = [&](int i) { ok = ok && wait(&sh.sempty[i], (sphases >> i & 1) ^ 1); };
        free_s(0);
        free_s(1);
        for (int j = 0; j < n && ok; ++j) {
          if (j == kLead) {
            free_s(4);
            free_s(5);
          }
          if (j >= kLead && (j & 2)) free_o();
          scores(q, place(j));
        }
        free_s(4);
        free_s(5);
        for (int j = 0; j < 2 && j < n; ++j) scores(q, j);
        if (n) {
          free_o();
          free_s(2);
          free_s(3);
        }
        for (int j = 0; j < n && ok; ++j) {
          const int g = j & 1;
          // The next scores go first: the group whose weights come now waits for nothing else.
          if (j + 2 < n) scores(q, g);
          ok = ok && wait(&sh.pfull[g], pphases >> g & 1) && wait(&sh.full[r.slot], r.phase);
          if (!ok) break;
          ptx::tc_fence_after();
          const uint32_t p = rows_lo(pbuf + g * 2 * kBlockBytes), v = rows_lo(ring + r.slot * kBlockBytes);
#pragma unroll
          for (int i = 0; i < 4; ++i) ptx::umma_i8_hl(o_hi, p + 2 * i, hi_128, v + 2 * i, hi_128, id_hi, j > 0 || i > 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) ptx::umma_i8_hl(o_lo, p + (kBlockBytes >> 4) + 2 * i, hi_128, v + 2 * i, hi_128, id_lo, j > 0 || i > 0);
          ptx::umma_commit(ptx::smem_u32(&sh.empty[r.slot]));
          ptx::umma_commit(ptx::smem_u32(&sh.pempty[g]));
          r.next(kRing);
          pphases ^= 1u << g;
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
  } else if (warp == 2) {
    // Units, and everything that is read to find out what to copy: blocks and their exponents, over the lanes.
    Finder finder;
    Ring ur;
    bool ok = true, more = true;
    for (int round = 0; ok && more; ++round, ur.next(kUnits)) {
      const int unit = round * (int)gridDim.x + ((round & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
      Unit u;
      more = finder.find(a, f, unit, lane, &u);
      if (!more) u.request = -1;
      ok = __all_sync(0xFFFFFFFFu, wait(&sh.uempty[ur.slot], ur.phase ^ 1));
      if (!ok) break;
      const int n = more ? u.b1 - u.b0 : 0;
      const int32_t* row = f.table + (long long)u.request * f.ldt + u.b0;
#pragma unroll 4
      for (int i = lane; i < n; i += 32) {
        const int id = row[i];
        const bool good = (unsigned)id < (unsigned)c.blocks;
        if (!good) atomicAdd(a.status + 1, 1u);
        const long long at = (long long)(good ? id : 0) * a.kv + u.head;
        sh.ids[ur.slot][i] = good ? id : -1;
        sh.exps[ur.slot][i] = (uint16_t)(min((int)c.k_exp[at], kAttnMaxExp) | min((int)c.v_exp[at], kAttnMaxExp) << 8 | (good ? 0 : kBad));
      }
      if (lane == 0) {
        sh.units[ur.slot] = u;
        if (more && u.tile == 0 && u.head == 0 && f.held[u.request] != u.held) atomicAdd(a.status + 1, 1u);
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.ufull[ur.slot]));
    }
  } else if (warp == 3) {
    // Queries: rows of D bytes into the layout of the MMA's operand.
    Ring qr, ur;
    Unit u;
    bool ok = true;
    for (; ok && __all_sync(0xFFFFFFFFu, take(ur, &u)); ur.next(kUnits), qr.next(2)) {
      ok = __all_sync(0xFFFFFFFFu, wait(&sh.qempty[qr.slot], qr.phase ^ 1));
      const Tile tile(a, u);
#pragma unroll 8
      for (int i = lane; ok && i < kRows * (D / 16); i += 32) {
        const int r = i / (D / 16), piece = i % (D / 16), flat = min(tile.flat0 + r, tile.flats - 1);     // rows behind the last one: any
        const long long row = u.row0 + flat / a.group;
        const int4 v = *reinterpret_cast<const int4*>(f.q8 + (row * a.heads + u.head * a.group + flat % a.group) * D + piece * 16);
        ptx::sts128(qbuf + qr.slot * kBlockBytes + swizzled(r, piece, D), v.x, v.y, v.z, v.w);
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
    const int w = (warp - 4) >> 3, half = (warp - 4) >> 2 & 1, part = (warp - 4) >> 2;   // group, half of a block's keys, both in one
    const int quarter = warp & 3, r = quarter * 32 + lane;                               // lanes of tensor memory, row of the tile
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16, s_mem = tmem + lanes + half * kHalf, words = table + lane * 4;
    const uint32_t p_hi = pbuf + w * 2 * kBlockBytes, p_lo = p_hi + kBlockBytes;
    Ring ur, orr;
    uint32_t sphases = 0, pphase = 1;
    Unit u;
    bool ok = true;
    // S may be written over: an arrival for each of the warps that share it in the second pass
    auto release = [&](int which, int arrivals) {
      ptx::tc_fence_before();
      __syncwarp();
      if (lane < arrivals) ptx::mbar_arrive(ptx::smem_u32(&sh.sempty[which]));
    };
    const uint32_t by_group = 65536 / a.group + 1;      // x / group = x * this >> 16 for x < 256, group <= 128
    for (;;) {
      // The two groups meet twice in a unit: here behind the first pass, whatever their other waits return (both leave, or none), and
      // behind the second. Then the first one stores the unit, and the other begins the next.
      const bool more = __all_sync(0xFFFFFFFFu, take(ur, &u));
      if (!more) u.b0 = u.b1 = u.len = u.tile = 0;
      const Tile tile(a, u);
      const int n = u.b1 - u.b0;
      const int rem0 = tile.flat0 % a.group, token0 = tile.flat0 / a.group;
      const int flat = tile.flat0 + r;
      const bool live = flat < tile.flats;
      const long long row = u.row0 + (live ? flat : tile.flat0) / a.group;
      const int head = u.head * a.group + flat % a.group;
      const Range see = visible(a, tile.position(a, u, live ? flat : tile.flat0), u.held);
      const int eq = live ? min((int)f.q_exp[row * a.heads + head], kAttnMaxExp) : 0;
      // blocks in [whole0, whole1) are seen whole by every row
      const Range low = visible(a, tile.position(a, u, tile.flat0), u.held), high = visible(a, tile.position(a, u, tile.flats - 1), u.held);
      const int whole0 = (high.first + kAttnBlock - 1) / kAttnBlock, whole1 = max(low.last, 0) / kAttnBlock;
      int T = INT32_MIN, V = 0;
      const int lead = min(n, kLead), rest = max(n - kLead, 0);
      bool leading = w == 1;
      int slot = leading ? 4 + half : w + 2 * half, j1 = leading ? half : kLead + slot;
      for (;; j1 += leading ? 2 : 4) {
        if (leading && j1 >= lead) {
          leading = false;
          slot = w + 2 * half;
          j1 = kLead + slot;
        }
        if (j1 >= n) break;
        const int j = j1;
        const int b = u.b0 + j, exps = sh.exps[ur.slot][j], W = sh.multipliers[eq + (exps & 255)];
        ok = ok && warp_wait(&sh.sfull[slot], sphases >> slot & 1);
        sphases ^= 1u << slot;
        if (!ok) break;
        ptx::tc_fence_after();
        int m[4] = {INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN};
        auto most = [&](auto masked) {
#pragma unroll
          for (int c0 = 0; c0 < kAttnBlock; c0 += 64) {
            uint32_t s0[32], s1[32];
            ptx::tmem_ld32(tmem + lanes + (slot & 3) * 128 + c0, s0);
            ptx::tmem_ld32(tmem + lanes + (slot & 3) * 128 + c0 + 32, s1);
            ptx::tmem_ld_wait32(s0);
            ptx::tmem_ld_wait32(s1);
            if (c0) release(slot, 2);
            const int first = see.first - b * kAttnBlock - c0, last = see.last - b * kAttnBlock - c0;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              if (masked.value) {
                m[i & 3] = i >= first && i < last ? max(m[i & 3], (int)s0[i]) : m[i & 3];
                m[i & 3] = i + 32 >= first && i + 32 < last ? max(m[i & 3], (int)s1[i]) : m[i & 3];
              } else {
                m[i & 3] = max(m[i & 3], max((int)s0[i], (int)s1[i]));
              }
            }
          }
        };
        if (b >= whole0 && b < whole1) most(std::false_type());
        else most(std::true_type());
        const int top = max(max(m[0], m[1]), max(m[2], m[3]));
        if (!(exps & kBad) && top != INT32_MIN) {
          T = max(T, score_octaves(top, W));
          V = max(V, exps >> 8 & 127);
        }
      }
      sh.top[part][r] = T;
      sh.vexp[part][r] = V;
      if (!ptx::all_agree(1, 32 * kSoft, more)) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        T = max(T, sh.top[i][r]);
        V = max(V, sh.vexp[i][r]);
      }
      // S 0 and 1 are read by all of a group from here on: what its other half has read counts, too
      const int other = w + 2 * (half ^ 1);
      sphases ^= (uint32_t)((rest - other + 3) >> 2 & (rest > other)) << other;
      long long L = 0;
      for (int j = w; j < n; j += 2) {
        const int b = u.b0 + j, exps = sh.exps[ur.slot][j], W = sh.multipliers[eq + (exps & 255)];
        const bool bad = exps & kBad, whole = b >= whole0 && b < whole1 && !bad;
        const int d = max(V - (exps >> 8 & 127), 0), C = -(T + 8192 * d);
        const int first = bad ? INT32_MAX : see.first - b * kAttnBlock - half * kHalf, last = see.last - b * kAttnBlock - half * kHalf;
        ok = ok && warp_wait(&sh.sfull[w], sphases >> w & 1);
        sphases ^= 1u << w;
        if (!ok) break;
        ptx::tc_fence_after();
        uint32_t sum = 0;
        uint32_t ahead[16];
        ptx::tmem_ld16(s_mem + w * 128, ahead);
#pragma unroll
        for (int c0 = 0; c0 < kHalf; c0 += 16) {
          uint32_t s[16];
          ptx::tmem_ld_wait16(ahead);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = ahead[i];
          if (c0 + 16 < kHalf) {                        // the next ones come while these are worked on
            ptx::tmem_ld16(s_mem + w * 128 + c0 + 16, ahead);
          } else {
            release(w, 1);
          }
          uint32_t hi[4], lo[4];
          auto weights = [&](auto masked) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              uint32_t x[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                int t = __viaddmax_s32(score_octaves((int)s[i + e], W), C, kWeightLow);
                if (masked.value) t = c0 + i + e >= first && c0 + i + e < last ? t : kWeightLow;
                x[e] = weight_bits(t, (int)ptx::lds32((uint32_t)(t & ((kWeightSegments - 1) << 7)) | words));
                sum += x[e];
              }
              split4(x, &hi[i / 4], &lo[i / 4]);
            }
          };
          if (whole) weights(std::false_type());
          else weights(std::true_type());
          if (c0 == 0) ok = warp_wait(&sh.pempty[w], pphase);           // the MMAs have read the weights before these
          const int piece = (half * kHalf + c0) / 16;
          ptx::sts128(p_hi + swizzled(r, piece, 128), hi[0], hi[1], hi[2], hi[3]);
          ptx::sts128(p_lo + swizzled(r, piece, 128), lo[0], lo[1], lo[2], lo[3]);
        }
        pphase ^= 1;
        ptx::fence_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.pfull[w]));
        L += (long long)(sum - kHalf * kWeightBias) << d;
      }
      sh.sum[part][r] = L;
      ptx::named_barrier(1, 32 * kSoft);
      if (w == 1) {
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.uempty[ur.slot]));
        ur.next(kUnits);
        continue;
      }
      L = sh.sum[0][r] + sh.sum[1][r] + sh.sum[2][r] + sh.sum[3][r];
      const Reciprocal rec = reciprocal(max(L, 1ll), V);
      constexpr int kLanes = D / 4, kAtOnce = 32 / kLanes, kRounds = kRows / (kSoft / 2 * kAtOnce);   // lanes of a row, rows of a warp
      const int piece = lane % kLanes;
      const int t0 = (warp - 4) * kAtOnce + lane / kLanes;
      auto head_of = [&](int t) { return u.head * a.group + rem0 + t - (int)((uint32_t)(rem0 + t) * by_group >> 16) * a.group; };
      int hd = head_of(t0);
      int4 rq[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) rq[e] = a.out[hd * D + piece * 4 + e];
      if (n) {
        ok = ok && warp_wait(&sh.ofull, orr.phase);
        orr.next(1);
        ptx::tc_fence_after();
      }
      // Quotients go through the weights' shared memory (all MMAs have read it), so that a warp then has rows whose elements lie side by
      // side: 16-byte piece c of row r at c ^ (r & 7).
#pragma unroll
      for (int c0 = half * (D / 2); c0 < (half + 1) * (D / 2); c0 += 8) {
        uint32_t h[8], l[8];
        ptx::tmem_ld8(o_hi + lanes + c0, h);
        ptx::tmem_ld8(o_lo + lanes + c0, l);
        ptx::tmem_ld_wait8(h);
        ptx::tmem_ld_wait8(l);
        int o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = L ? quotient((int)h[i], (int)l[i], rec) : 0;
#pragma unroll
        for (int i = 0; i < 8; i += 4)
          ptx::sts128(pbuf + r * (4 * D) + ((((c0 + i) >> 2) ^ (r & 7)) << 4), (uint32_t)o[i], (uint32_t)o[i + 1], (uint32_t)o[i + 2], (uint32_t)o[i + 3]);
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0 && n) ptx::mbar_arrive(ptx::smem_u32(&sh.oempty));
      ptx::named_barrier(2, 16 * kSoft);
      constexpr int kStep = kSoft / 2 * kAtOnce;                       // rows of the eight warps together
      const uint8_t* const piece_at = smem + (pbuf - table);
      auto quotients = [&](int t) { return *reinterpret_cast<const int4*>(piece_at + t * (4 * D) + ((piece ^ (t & 7)) << 4)); };
      if (f.vector && a.y_full && kStep % a.group == 0 && tile.flats - tile.flat0 == kRows && ok) {
        // Rows of a warp have one head, tokens at one distance, and the outputs' clip is the type's: 8-bit outputs in words.
        int8_t* p = (int8_t*)f.y + (long long)(u.row0 + token0 + (int)((uint32_t)(rem0 + t0) * by_group >> 16)) * f.ldy + hd * D + piece * 4;
        const long long step = (long long)(kStep / a.group) * f.ldy;
#pragma unroll
        for (int i = 0; i < kRounds; ++i, p += step) {
          const int4 o = quotients(t0 + i * kStep);
          *reinterpret_cast<uint32_t*>(p) = packed(requantised(o.x, rq[0]), requantised(o.y, rq[1]), requantised(o.z, rq[2]), requantised(o.w, rq[3]));
        }
      } else {
#pragma unroll 1
        for (int i = 0; i < kRounds && ok; ++i) {
          const int t = t0 + i * kStep, at = head_of(t);
          if (at != hd) {
            hd = at;
#pragma unroll
            for (int k = 0; k < 4; ++k) rq[k] = a.out[hd * D + piece * 4 + k];
          }
          if (tile.flat0 + t >= tile.flats) break;
          const int4 o = quotients(t);
          const int y[4] = {clipped(requantised(o.x, rq[0]), a.lo, a.hi), clipped(requantised(o.y, rq[1]), a.lo, a.hi),
                            clipped(requantised(o.z, rq[2]), a.lo, a.hi), clipped(requantised(o.w, rq[3]), a.lo, a.hi)};
          const long long to = (long long)(u.row0 + token0 + (int)((uint32_t)(rem0 + t) * by_group >> 16)) * f.ldy + hd * D + piece * 4;
          if (a.y_bytes == 1) {
            int8_t* p = (int8_t*)f.y + to;
            if (f.vector) {
              *reinterpret_cast<uint32_t*>(p) = __byte_perm(__byte_perm((uint32_t)y[0], (uint32_t)y[1], 0x0040),
                                                            __byte_perm((uint32_t)y[2], (uint32_t)y[3], 0x0040), 0x5410);
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k) p[k] = (int8_t)y[k];
            }
          } else {
            int* p = (int*)f.y + to;
            if (f.vector) {
              *reinterpret_cast<int4*>(p) = make_int4(y[0], y[1], y[2], y[3]);
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k) p[k] = y[k];
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.uempty[ur.slot]));
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
