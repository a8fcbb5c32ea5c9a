// Attention of few rows (include/iodf.h: iodf_attn_forward): the next tokens of requests with long contexts.
//
// A unit of work is up to 16 rows ((token, query head) pairs) of a request and the keys of one head of the cache. The keys are the
// MMA's M and the rows its N, so that K and V go from the copy's shared memory straight into the tensor cores:
//   S^T [128 keys][16] = K q^T,   O^T [dim][16] += V^T p^T
// and a thread of the softmax owns a key. K is read first and its scores stay where they are, in tensor memory, until the largest of all
// is known (26 blocks; t of further ones lies in shared memory, and where that is full K is read again), then V. What bounds it is the
// reading of K and V, once each.
//
// Work is spread in teams: a request's blocks go to 1, 2, 4 or 8 CTAs of a cluster, by their number; teams that are smaller than a
// cluster share it. CTAs of a team tell each other their largest t and, at the end, their sums, each CTA the owners of the dimensions,
// through the cluster's shared memory. Clusters are persistent and take the large teams first; copies run ahead into the next unit.
// Where units are fewer than clusters, a cluster is one team and as large as still lets all units run at once.
//
// Measured, 32 query heads of 128 over 8: one token after 1000 12.2 us, a chain of steps of which none fills anything (units found, K and
// its scores, the team's largest t, V, the team's sums, outputs); 64 requests of up to 8192 tokens 35 us, 69 MB at 1.9 TB/s, contexts
// that differ and the same chain; one token after 131072 74 us, 268 MB at 3.6 TB/s, scores, weights and their MMAs of one CTA behind one another
// (scores read back and kept in words 291, kept in tensor memory 121, twice the weights' room 116, scores computed again ahead of the values 93,
// teams as large as the GPU holds 75).
#include <algorithm>

#include "../../include/iodf.h"
#include "attn_device.cuh"
#include "attn_kernels.h"
#include "iodf_dev.h"
#include "ptx_attn.cuh"

namespace iodf {
namespace {

constexpr int kN = 16;                   // of the scores' MMAs, the least; a unit has up to 4, 8 or 16 rows
constexpr int kUnitsS = 3;
constexpr int kAhead = 3;                // blocks that scores computed a second time are ahead of the values
constexpr int kTileBytes = 16384;        // of a slot: 128 rows of up to 128 bytes; V^T is read as 128 rows whatever the dimension
constexpr int kLeastCluster = 8, kMaxTeam = kAttnMaxTeam, kClasses = 5;             // teams of 1, 2, 4, 8; of a whole cluster
constexpr int kMaxPart = kAttnMaxBlocks / kLeastCluster;          // blocks of one CTA
constexpr int kMaxChunks = kAttnSplitRequests / 32;

// Dimensions of a row's output that one CTA of a team finishes. The last CTAs may have fewer, or none.
__host__ __device__ constexpr int owned(int dim, int team) { return (dim + team - 1) / team; }
// Places of a CTA's sums: each member of the team has `owned` of them, also where dimensions do not divide evenly (10 CTAs, 128 dimensions: 130).
constexpr int most_places(int dim, int least, int most) {
  int places = 0;
  for (int team = least; team <= most; ++team) places = team * owned(dim, team) > places ? team * owned(dim, team) : places;
  return places;
}
constexpr int kPlaces = 128, kPlacesBig = 140;           // teams of 1, 2, 4, 8; of up to 16
static_assert(most_places(128, 1, 1) <= kPlaces && most_places(128, 2, 2) <= kPlaces && most_places(128, 4, 4) <= kPlaces && most_places(128, 8, 8) <= kPlaces, "teams within a cluster");
static_assert(most_places(32, 1, kMaxTeam) <= kPlacesBig && most_places(64, 1, kMaxTeam) <= kPlacesBig && most_places(128, 1, kMaxTeam) <= kPlacesBig, "teams as large as a cluster");

// Two shapes: one CTA to an SM, with room for the scores of many blocks, or two, so that one unit's waits are another's work.
//   weights: hi = (p + 128) >> 8 and the low byte of p + 128, which is 128 more than lo; both are unsigned, so one MMA has rows of hi, rows of
//   lo and a row of ones, whose product (the sum of v) takes the 128 off again. 16 rows need two MMAs: hi, and lo signed.
template <int kCols, int kGroups>
struct Shape {
  static constexpr int kThreads = 128 + 128 * kGroups, kWarps = kThreads / 32, kSoft = 4 * kGroups;     // warp 0 copies, 1 MMAs, 2 units, 3 queries, then softmax
  static constexpr bool kBig = kGroups == 4;
  static constexpr int kRing = kBig ? 5 : 3, kColumns = kBig ? 512 : 256;                               // stages; of tensor memory
  static constexpr int kO = kCols == 4 ? 16 : 32;                                                      // of O: N of its MMAs, or twice 16
  static constexpr int kScores = (kColumns - 32) / kN, kHeld = kScores - 4;      // S: of the first blocks they stay, the last four take turns
  static constexpr int kSumPlaces = kBig ? kPlacesBig : kPlaces;
  static constexpr int kDynamic = (kBig ? 200 : 86) * 1024 + (kSumPlaces - 128) * 16 * 8;               // the same for all kCols
  static constexpr int kOperand = kCols > 4 ? 4096 : 2048;                                             // of weights: rows of 128 bytes
  static constexpr int kQBytes = kCols > 8 ? 2048 : 1024;                                              // of queries; MMAs read 16 rows, the others may be anything
  static constexpr int kP = kRing * kTileBytes, kQ = kP + 2 * kGroups * kOperand, kSums = kQ + 2 * kQBytes + 1024;
  static constexpr int kKept = kSums + kSumPlaces * kCols * 8;
  static constexpr int kKeptBlocks = (kDynamic - 1024 - kKept) / (kCols * 512) > 0 ? (kDynamic - 1024 - kKept) / (kCols * 512) : 0;      // t of 128 keys, 32 bits
  static constexpr int kKeep = kHeld + kKeptBlocks;
  static_assert(kKept + 1024 <= kDynamic, "shared memory");
};

struct UnitS {
  int request, head, row0, len;
  int flat0, cols;                       // rows of the unit: [flat0, flat0 + cols)
  int held, b0, n;                       // this CTA's blocks: [b0, b0 + n)
  int cls, team, member;                 // CTAs, and which of them
};

template <class Sh>
struct SharedS {
  uint64_t full[Sh::kRing], empty[Sh::kRing], sfull[Sh::kScores], sempty[Sh::kScores], pfull[Sh::kWarps], pempty[Sh::kWarps], qfull[2], qempty[2];
  uint64_t ofull, oempty, ufull[kUnitsS], efull[kUnitsS], uempty[kUnitsS], tops[kClasses], sums[kClasses];
  uint32_t abort_flag, tmem;
  int total[kClasses];                   // units of each class
  UnitS units[kUnitsS];
  int ids[kUnitsS][kMaxPart];            // blocks; -1: outside the cache, nobody sees it
  uint8_t ek[kUnitsS][kMaxPart], ev[kUnitsS][kMaxPart];
  int top[Sh::kSoft][kN], vexp[Sh::kSoft][kN];           // of the softmax warps
  long long sum[Sh::kSoft][kN];
  int vtop[kN];                          // V of each row, over the team
  int team_top[kMaxTeam][kN], team_vexp[kMaxTeam][kN];
  long long team_sum[kMaxTeam][kN];
};

struct SplitArgs {
  int cluster, per_cta;                  // CTAs of a cluster; blocks that one CTA takes before the team grows
  int one_team;                          // a cluster is a team
  int chunks;                            // of 32 requests
};

struct RingS {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int size) {
    if (++slot == size) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

// What a request asks for: its rows, its units of each cache head, the class of its teams.
struct Ask {
  int start, len, held, tiles, cls;
  __device__ __forceinline__ Ask(const AttnArgs& a, const ForwardArgs& f, const SplitArgs& s, int cols, int q)
      : start(0), len(0), held(0), tiles(0), cls(0) {
    if (q >= f.n) return;
    const int s0 = f.row_start[q], s1 = f.row_start[q + 1];
    held = min(max(f.held[q], 0), f.width * kAttnBlock);
    start = min(max(s0, 0), f.rows);
    len = max(min(max(s1, 0), f.rows) - start, 0);
    tiles = (len * a.group + cols - 1) / cols;
    const int first = visible(a, held - len, held).first / kAttnBlock, blocks = (held + kAttnBlock - 1) / kAttnBlock - first;
    if (s.one_team) cls = kClasses - 1;
    else while (s.cluster >> (cls + 1) && blocks > s.per_cta << cls) ++cls;
  }
};

template <int D, int kCols, int kGroups>
__global__ void __launch_bounds__(128 + 128 * kGroups, kGroups == 4 ? 1 : 2) split_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                                                             const AttnArgs a, const CacheArgs c, const ForwardArgs f, const SplitArgs s) {
  typedef Shape<kCols, kGroups> At;
  constexpr int kThreadsS = At::kThreads, kWarpsS = At::kWarps, kSoft = At::kSoft, kRingS = At::kRing, kScores = At::kScores, kHeld = At::kHeld,
                kKeep = At::kKeep, kBuffers = 2 * kGroups;
  extern __shared__ uint8_t raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  __shared__ SharedS<At> sh;
  __shared__ int table[kWeightSegments * 32];           // a copy for each lane: no bank is asked twice
  __shared__ int before[kClasses][kMaxChunks + 1];      // units of each class before a chunk of 32 requests
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = ptx::smem_u32(smem), pbuf = ring + At::kP, qbuf = ring + At::kQ, osum = ring + At::kSums;
  const int* const osums = reinterpret_cast<const int*>(smem + At::kSums);
  int* const kept = reinterpret_cast<int*>(smem + At::kKept);
  volatile uint32_t* const abort_flag = &sh.abort_flag;
  const int rank = (int)ptx::cluster_rank();
  if (tid == 0) {
    auto init = [](uint64_t* bars, int n, int count) {
      for (int i = 0; i < n; ++i) ptx::mbar_init(ptx::smem_u32(bars + i), count);
    };
    init(sh.full, kRingS, 1);
    init(sh.empty, kRingS, 1);
    init(sh.sfull, kScores, 1);
    init(sh.sempty, kScores, 4);
    init(sh.pfull, kBuffers, 4);
    init(sh.pempty, kBuffers, 1);
    init(sh.qfull, 2, 1);
    init(sh.qempty, 2, 1);
    init(&sh.ofull, 1, 1);
    init(&sh.oempty, 1, kSoft);
    init(sh.ufull, kUnitsS, 1);
    init(sh.efull, kUnitsS, 1);
    init(sh.uempty, kUnitsS, 3 + kSoft);
    for (int i = 0; i < kClasses; ++i) {
      init(&sh.tops[i], 1, i == kClasses - 1 ? s.cluster : 1 << i);
      init(&sh.sums[i], 1, i == kClasses - 1 ? s.cluster : 1 << i);
    }
    ptx::mbar_init_fence();
    sh.abort_flag = 0;
  }
  ptx::cluster_arrive();                                // every CTA runs, its barriers are set up
  if (warp == 2) ptx::tmem_alloc(ptx::smem_u32(&sh.tmem), At::kColumns);
  for (int i = tid; i < kWeightSegments * 32; i += kThreadsS) table[i] = weight_word(i / 32);
  if (kCols < 16)                                       // the rows of ones
    for (int i = tid; i < kBuffers * 32; i += kThreadsS)
      reinterpret_cast<uint32_t*>(smem + At::kP + i / 32 * At::kOperand + 2 * kCols * 128)[i % 32] = 0x01010101u;
  ptx::fence_async_smem();
  const Ask first(a, f, s, kCols, warp == 2 ? lane : f.n);          // warp 2 has the first requests at hand when it looks for units
  for (int k = (warp + kWarpsS - 2) % kWarpsS; k < s.chunks; k += kWarpsS) {
    const Ask ask = k ? Ask(a, f, s, kCols, k * 32 + lane) : first;
#pragma unroll
    for (int i = 0; i < kClasses; ++i) {
      const int n = __reduce_add_sync(0xFFFFFFFFu, ask.cls == i ? ask.tiles * a.kv : 0);
      if (lane == 0) before[i][k + 1] = n;
    }
  }
  ptx::cluster_wait();
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (warp < kClasses) {                                // prefix sums over the chunks
    int sum = 0;
    for (int k0 = 0; k0 < s.chunks; k0 += 32) {
      int v = k0 + lane < s.chunks ? before[warp][k0 + lane + 1] : 0;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int o = __shfl_up_sync(0xFFFFFFFFu, v, d);
        if (lane >= d) v += o;
      }
      if (k0 + lane < s.chunks) before[warp][k0 + lane + 1] = sum + v;
      sum += __shfl_sync(0xFFFFFFFFu, v, 31);
    }
    if (lane == 0) {
      before[warp][0] = 0;
      sh.total[warp] = sum;
    }
  }
  __syncthreads();
  const uint32_t tmem = sh.tmem, o_mem = tmem + kScores * kN;
  auto wait = [&](uint64_t* bar, uint32_t phase) { return ptx::quick_wait(abort_flag, a.status, bar, phase, kSpinLimit); };
  auto warp_wait = [&](uint64_t* bar, uint32_t phase) { return __all_sync(0xFFFFFFFFu, wait(bar, phase)) != 0; };
  auto take = [&](const RingS& r, UnitS* u) {
    if (!wait(&sh.ufull[r.slot], r.phase)) return false;
    *u = sh.units[r.slot];
    return u->request >= 0;
  };
  // for what other CTAs have written before they arrived
  auto team_wait = [&](uint64_t* bar, uint32_t phase) {
    if (!warp_wait(bar, phase)) return false;
    ptx::mbar_acquire_cluster(ptx::smem_u32(bar), phase);
    return true;
  };
  // of blocks from kKeep on the scores are computed twice
  // where the scores of the unit's block i are: all of a call's uses of a slot are counted in bits, one for each
  auto buffer_of = [](int i) { return 2 * (i % kGroups) + (i / kGroups & 1); };     // of weights, two for each group
  auto slot_of = [](int i) { return i < kHeld ? i : kHeld + (i - kHeld) % (kScores - kHeld); };

  if (warp == 0) {
    if (ptx::elect_one()) {
      RingS r, ur;
      UnitS u;
      bool ok = true;
      auto copy = [&](const CUtensorMap* map, int row, int count) {
        ok = ok && wait(&sh.empty[r.slot], r.phase ^ 1);
        if (!ok) return;
        const uint32_t bar = ptx::smem_u32(&sh.full[r.slot]);
        ptx::mbar_expect_tx(bar, kAttnBlock * D);
        ptx::tile_g2s(ring + r.slot * kTileBytes, map, 0, row, bar);
        r.next(kRingS);
      };
      for (; ok && take(ur, &u); ur.next(kUnitsS)) {
        const int* ids = sh.ids[ur.slot];
        for (int i = 0; i < u.n && ok; ++i) copy(&kmap, (max(ids[i], 0) * a.kv + u.head) * kAttnBlock, D);
        for (int i = -kAhead; i < u.n && ok; ++i) {
          if (i + kAhead >= kKeep && i + kAhead < u.n) copy(&kmap, (max(ids[i + kAhead], 0) * a.kv + u.head) * kAttnBlock, D);
          if (i >= 0) copy(&vmap, (max(ids[i], 0) * a.kv + u.head) * D, D);
        }
        ptx::mbar_arrive(ptx::smem_u32(&sh.uempty[ur.slot]));
      }
      for (int i = 0; ok && i < kRingS; ++i, r.next(kRingS)) ok = wait(&sh.empty[r.slot], r.phase ^ 1);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (ptx::elect_one()) {
      constexpr uint32_t id_s = idesc_i8(128, kN, false, false), id_lo = idesc_i8(128, 16, false, false);
      constexpr uint32_t id_p = idesc_i8(128, kCols == 16 ? 16 : At::kO, false, true);
      constexpr uint32_t hi_d = rows_hi(D), hi_128 = rows_hi(128);
      RingS r, ur, qr, orr;
      uint32_t pphases = 0, sphases = 0;
      UnitS u;
      bool ok = true;
      auto scores = [&](uint32_t q, int slot) {
        ok = ok && wait(&sh.full[r.slot], r.phase) && wait(&sh.sempty[slot], (sphases >> slot & 1) ^ 1);
        if (!ok) return;
        ptx::tc_fence_after();
        const uint32_t k = rows_lo(ring + r.slot * kTileBytes);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) ptx::umma_i8_hl(tmem + slot * kN, k + 2 * i, hi_d, q + 2 * i, hi_d, id_s, i > 0);
        ptx::umma_commit(ptx::smem_u32(&sh.empty[r.slot]));
        ptx::umma_commit(ptx::smem_u32(&sh.sfull[slot]));
        r.next(kRingS);
        sphases ^= 1u << slot;
      };
      for (; ok && take(ur, &u); ur.next(kUnitsS)) {
        ok = wait(&sh.qfull[qr.slot], qr.phase);
        ptx::tc_fence_after();
        const uint32_t q = rows_lo(qbuf + qr.slot * At::kQBytes);
        for (int i = 0; i < u.n && ok; ++i) scores(q, slot_of(i));
        for (int i = -kAhead; i < u.n && ok; ++i) {
          if (i + kAhead >= kKeep && i + kAhead < u.n) scores(q, slot_of(i + kAhead));
          if (i < 0) continue;
          const int g = buffer_of(i);
          if (i == 0) ok = ok && wait(&sh.oempty, orr.phase ^ 1);
          ok = ok && wait(&sh.pfull[g], pphases >> g & 1) && wait(&sh.full[r.slot], r.phase);
          if (!ok) break;
          ptx::tc_fence_after();
          const uint32_t v = rows_lo(ring + r.slot * kTileBytes), p = rows_lo(pbuf + g * At::kOperand);
#pragma unroll
          for (int k = 0; k < 4; ++k) ptx::umma_i8_hl(o_mem, v + 2 * k, hi_128, p + 2 * k, hi_128, id_p, i > 0 || k > 0);
          if (kCols == 16) {
#pragma unroll
            for (int k = 0; k < 4; ++k) ptx::umma_i8_hl(o_mem + 16, v + 2 * k, hi_128, p + (2048 >> 4) + 2 * k, hi_128, id_lo, i > 0 || k > 0);
          }
          ptx::umma_commit(ptx::smem_u32(&sh.empty[r.slot]));
          ptx::umma_commit(ptx::smem_u32(&sh.pempty[g]));
          pphases ^= 1u << g;
          r.next(kRingS);
        }
        if (ok && u.n) {
          ptx::umma_commit(ptx::smem_u32(&sh.ofull));
          orr.next(1);
        }
        if (ok) ptx::umma_commit(ptx::smem_u32(&sh.qempty[qr.slot]));
        qr.next(2);
        ptx::mbar_arrive(ptx::smem_u32(&sh.uempty[ur.slot]));
      }
      for (int i = 0; ok && i < kBuffers; ++i) ok = wait(&sh.pempty[i], (pphases >> i & 1) ^ 1);
    }
    __syncwarp();
  } else if (warp == 2) {
    // Units: items of the cluster, class by class from the largest teams on; in one item a cluster's CTAs work in teams of one size.
    RingS ur;
    bool ok = true;
    const int clusters = (int)gridDim.x / s.cluster;
    int item = (int)blockIdx.x / s.cluster;
    for (int cls = kClasses - 1; cls >= 0 && ok; --cls) {
      const int team = cls == kClasses - 1 ? s.cluster : 1 << cls, teams = max(1, s.cluster / team);
      const int items = (sh.total[cls] + teams - 1) / teams;
      for (; item < items && ok; item += clusters) {
        const int unit = item * teams + rank / team;
        if (unit >= sh.total[cls]) continue;
        int lo = 0, hi = s.chunks - 1;                  // the chunk that holds it
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (before[cls][mid + 1] > unit) hi = mid;
          else lo = mid + 1;
        }
        const Ask ask = lo ? Ask(a, f, s, kCols, lo * 32 + lane) : first;
        const int mine = ask.cls == cls ? ask.tiles * a.kv : 0;
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
          const int o = __shfl_up_sync(0xFFFFFFFFu, upto, d);
          if (lane >= d) upto += o;
        }
        const int in = unit - before[cls][lo];
        const int from = __ffs((int)__ballot_sync(0xFFFFFFFFu, in < upto)) - 1;
        UnitS u;
        u.request = lo * 32 + from;
        u.row0 = __shfl_sync(0xFFFFFFFFu, ask.start, from);
        u.len = __shfl_sync(0xFFFFFFFFu, ask.len, from);
        u.held = __shfl_sync(0xFFFFFFFFu, ask.held, from);
        const int theirs = __shfl_sync(0xFFFFFFFFu, mine, from), at = in - (__shfl_sync(0xFFFFFFFFu, upto, from) - theirs);
        if ((unsigned)at >= (unsigned)theirs) {         // requests that share rows, more of them than can be counted
          cls = 0;
          break;
        }
        u.head = at % a.kv;
        u.flat0 = at / a.kv * kCols;
        u.cols = min(kCols, u.len * a.group - u.flat0);
        u.cls = cls;
        u.team = team;
        u.member = rank % team;
        const Range low = visible(a, u.held - u.len + u.flat0 / a.group, u.held);
        const Range high = visible(a, u.held - u.len + (u.flat0 + u.cols - 1) / a.group, u.held);
        const int b0 = low.first / kAttnBlock, n = high.last <= low.first ? 0 : (high.last + kAttnBlock - 1) / kAttnBlock - b0;
        u.b0 = b0 + u.member * n / u.team;
        u.n = b0 + (u.member + 1) * n / u.team - u.b0;
        ok = __all_sync(0xFFFFFFFFu, wait(&sh.uempty[ur.slot], ur.phase ^ 1));
        if (!ok) break;
        for (int i = lane; i < u.n; i += 32) {
          const int id = f.table[(long long)u.request * f.ldt + u.b0 + i];
          const bool good = (unsigned)id < (unsigned)c.blocks;
          if (!good) atomicAdd(a.status + 1, 1u);
          sh.ids[ur.slot][i] = good ? id : -1;
        }
        if (lane == 0) {
          sh.units[ur.slot] = u;
          if (u.flat0 == 0 && u.head == 0 && u.member == 0 && f.held[u.request] != u.held) atomicAdd(a.status + 1, 1u);
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.ufull[ur.slot]));
        for (int i = lane; i < u.n; i += 32) {          // needed later than the blocks themselves
          const long long e = (long long)max(sh.ids[ur.slot][i], 0) * a.kv + u.head;
          sh.ek[ur.slot][i] = (uint8_t)min((int)c.k_exp[e], kAttnMaxExp);
          sh.ev[ur.slot][i] = (uint8_t)min((int)c.v_exp[e], kAttnMaxExp);
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.efull[ur.slot]));
        ur.next(kUnitsS);
      }
      item -= items;                                    // of the next class
    }
    ok = ok && __all_sync(0xFFFFFFFFu, wait(&sh.uempty[ur.slot], ur.phase ^ 1));
    if (ok && lane == 0) {
      sh.units[ur.slot].request = -1;
      ptx::mbar_arrive(ptx::smem_u32(&sh.ufull[ur.slot]));
    }
    __syncwarp();
  } else if (warp == 3) {
    RingS ur, qr;
    UnitS u;
    bool ok = true;
    for (; ok && __all_sync(0xFFFFFFFFu, take(ur, &u)); ur.next(kUnitsS), qr.next(2)) {
      ok = __all_sync(0xFFFFFFFFu, wait(&sh.qempty[qr.slot], qr.phase ^ 1));
      for (int i = lane; ok && i < u.cols * (D / 16); i += 32) {
        const int r = i / (D / 16), piece = i % (D / 16), flat = u.flat0 + r;
        const long long row = u.row0 + flat / a.group;
        const int4 v = *reinterpret_cast<const int4*>(f.q8 + (row * a.heads + u.head * a.group + flat % a.group) * D + piece * 16);
        ptx::sts128(qbuf + qr.slot * At::kQBytes + swizzled(r, piece, D), v.x, v.y, v.z, v.w);
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
    const int w = (warp - 4) >> 2, quarter = warp & 3, key = quarter * 32 + lane, me = warp - 4;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    RingS ur, orr;
    uint32_t pphases = 0, team_phases = 0, sphases = 0;
    UnitS u;
    bool ok = true;
    while (ptx::all_agree(1, 32 * kSoft, take(ur, &u))) {
      const int nc = u.cols;
      // lane c < cols has the constants of row c
      const int flat = u.flat0 + min(lane, nc - 1);
      const long long row = u.row0 + flat / a.group;
      const int head = u.head * a.group + flat % a.group;
      const Range see = visible(a, u.held - u.len + flat / a.group, u.held);
      const int eq = min((int)f.q_exp[row * a.heads + head], kAttnMaxExp);
      const int whole0 = (__reduce_max_sync(0xFFFFFFFFu, see.first) + kAttnBlock - 1) / kAttnBlock;
      const int whole1 = max(__reduce_min_sync(0xFFFFFFFFu, see.last), 0) / kAttnBlock;
      int T = INT32_MIN, V = 0;                         // of row `lane`
      // t of the keys of block i from S, lowest where it is not seen
      auto octaves = [&](int i, int (&t)[kCols]) {
        uint32_t x[kCols];
        if constexpr (kCols == 4) ptx::tmem_ld4(tmem + lanes + slot_of(i) * kN, x);
        else if constexpr (kCols == 8) ptx::tmem_ld8(tmem + lanes + slot_of(i) * kN, x);
        else ptx::tmem_ld16(tmem + lanes + slot_of(i) * kN, x);
        const int b = u.b0 + i, k = b * kAttnBlock + key;
        const int W = score_multiplier(a.score_m0, eq + sh.ek[ur.slot][i], a.score_s);
        const bool bad = sh.ids[ur.slot][i] < 0, whole = b >= whole0 && b < whole1 && !bad;
        if constexpr (kCols == 4) ptx::tmem_ld_wait4(x);
        else if constexpr (kCols == 8) ptx::tmem_ld_wait8(x);
        else ptx::tmem_ld_wait16(x);
#pragma unroll
        for (int e = 0; e < kCols; ++e) t[e] = score_octaves((int)x[e], __shfl_sync(0xFFFFFFFFu, W, e));
        if (!whole) {
#pragma unroll
          for (int e = 0; e < kCols; ++e) {
            const int first = __shfl_sync(0xFFFFFFFFu, see.first, e), last = __shfl_sync(0xFFFFFFFFu, see.last, e);
            if (bad || k < first || k >= last) t[e] = INT32_MIN;
          }
        }
        return whole;
      };
      auto release = [&](int i) {                       // S of block i may be written over
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.sempty[slot_of(i)]));
      };
      ok = ok && warp_wait(&sh.efull[ur.slot], ur.phase);
      int tops[kCols];
#pragma unroll
      for (int e = 0; e < kCols; ++e) tops[e] = INT32_MIN;
      for (int i = w; i < u.n && ok; i += kGroups) {
        ok = warp_wait(&sh.sfull[slot_of(i)], sphases >> slot_of(i) & 1);
        if (!ok) break;
        ptx::tc_fence_after();
        int t[kCols];
        const bool whole = octaves(i, t);
        if (i >= kHeld) {
          release(i);
          sphases ^= 1u << slot_of(i);
        }
        if (whole) V = max(V, (int)sh.ev[ur.slot][i]);
#pragma unroll
        for (int e = 0; e < kCols; ++e) {
          tops[e] = max(tops[e], t[e]);
          if (!whole && __any_sync(0xFFFFFFFFu, t[e] != INT32_MIN) && lane == e) V = max(V, (int)sh.ev[ur.slot][i]);
          if (i >= kHeld && i < kKeep) kept[((i - kHeld) * kCols + e) * kAttnBlock + key] = t[e];
        }
      }
#pragma unroll
      for (int e = 0; e < kCols; ++e) {
        const int top = __reduce_max_sync(0xFFFFFFFFu, tops[e]);
        if (lane == e) T = top;
      }
      if (lane < kCols) {
        sh.top[me][lane] = T;
        sh.vexp[me][lane] = V;
      }
      ptx::named_barrier(1, 32 * kSoft);
#pragma unroll
      for (int i = 0; i < kSoft; ++i) {
        T = max(T, sh.top[i][lane & (kCols - 1)]);
        V = max(V, sh.vexp[i][lane & (kCols - 1)]);
      }
      if (u.team > 1) {
        if (me == 0) {
          const uint32_t to = (uint32_t)(rank - u.member + min(lane, u.team - 1));
          const uint32_t top = ptx::cluster_addr(ptx::smem_u32(&sh.team_top[u.member][0]), to);
          const uint32_t vexp = ptx::cluster_addr(ptx::smem_u32(&sh.team_vexp[u.member][0]), to);
          for (int e = 0; e < nc; ++e) {
            const int t = __shfl_sync(0xFFFFFFFFu, T, e), v = __shfl_sync(0xFFFFFFFFu, V, e);
            if (lane < u.team) {
              ptx::st_cluster(top + 4 * e, (uint32_t)t);
              ptx::st_cluster(vexp + 4 * e, (uint32_t)v);
            }
          }
          if (lane < u.team) ptx::mbar_arrive_cluster(ptx::cluster_addr(ptx::smem_u32(&sh.tops[u.cls]), to));
          __syncwarp();
        }
        ok = ok && team_wait(&sh.tops[u.cls], team_phases >> u.cls & 1);
        for (int m = 0; m < u.team; ++m) {
          T = max(T, sh.team_top[m][lane & (kCols - 1)]);
          V = max(V, sh.team_vexp[m][lane & (kCols - 1)]);
        }
      }
      if (me == 0 && lane < kCols) sh.vtop[lane] = V;
      long long Ls[kCols];
#pragma unroll
      for (int e = 0; e < kCols; ++e) Ls[e] = 0;
      for (int i = w; i < u.n && ok; i += kGroups) {
        const int buffer = buffer_of(i);
        const uint32_t p_hi = pbuf + buffer * At::kOperand, p_lo = p_hi + kCols * 128;
        ok = warp_wait(&sh.pempty[buffer], (pphases >> buffer & 1) ^ 1) && (i < kKeep || warp_wait(&sh.sfull[slot_of(i)], sphases >> slot_of(i) & 1));
        pphases ^= 1u << buffer;
        if (!ok) break;
        ptx::tc_fence_after();
        const int below = max(V - sh.ev[ur.slot][i], 0), off = -(T + 8192 * below);
        int t[kCols];
        if (i < kHeld || i >= kKeep) {
          octaves(i, t);
          release(i);
          sphases ^= 1u << slot_of(i);
        } else {
#pragma unroll
          for (int e = 0; e < kCols; ++e) t[e] = kept[((i - kHeld) * kCols + e) * kAttnBlock + key];
        }
#pragma unroll
        for (int e = 0; e < kCols; ++e) {
          const int down = __shfl_sync(0xFFFFFFFFu, off, e), by = __shfl_sync(0xFFFFFFFFu, below, e);
          const int n = t[e] == INT32_MIN ? kWeightLow : max(t[e] + down, kWeightLow);
          const uint32_t x = weight_bits(n, *reinterpret_cast<const int*>(reinterpret_cast<const char*>(table) + ((n & ((kWeightSegments - 1) << 7)) | lane * 4)));
          const uint32_t at = (uint32_t)(e * 128 + (((key >> 4) ^ (e & 7)) << 4) + (key & 15));
          const uint32_t at_lo = (uint32_t)(e * 128 + (((key >> 4) ^ ((e + kCols) & 7)) << 4) + (key & 15));
          asm volatile("st.shared.u8 [%0], %1;" ::"r"(p_hi + at), "r"(x >> 8) : "memory");
          asm volatile("st.shared.u8 [%0], %1;" ::"r"(p_lo + at_lo), "r"(kCols == 16 ? x ^ 0x80u : x) : "memory");
          Ls[e] += (x - kWeightBias) << by;             // below 2^28
        }
        ptx::tc_fence_before();
        ptx::fence_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.pfull[buffer]));
      }
      long long L = 0;                                  // of row `lane`
#pragma unroll
      for (int e = 0; e < kCols; ++e) {                 // below 2^35 in a thread: summed in two parts
        const uint32_t low = __reduce_add_sync(0xFFFFFFFFu, (uint32_t)(Ls[e] & 0xFFFFF)), high = __reduce_add_sync(0xFFFFFFFFu, (uint32_t)(Ls[e] >> 20));
        if (lane == e) L = ((long long)high << 20) + low;
      }
      if (lane < kCols) sh.sum[me][lane] = L;
      ptx::named_barrier(1, 32 * kSoft);
      L = 0;
#pragma unroll
      for (int i = 0; i < kSoft; ++i) L += sh.sum[i][lane & (kCols - 1)];
      uint32_t hi[kCols], lo[kCols];
#pragma unroll
      for (int e = 0; e < kCols; ++e) hi[e] = lo[e] = 0;
      if (u.n) {
        ok = ok && warp_wait(&sh.ofull, orr.phase);
        orr.next(1);
        ptx::tc_fence_after();
        if (ok) {
          uint32_t x[16];
          ptx::tmem_ld16(o_mem + lanes, x);
          ptx::tmem_ld_wait16(x);
          if constexpr (kCols == 16) {
#pragma unroll
            for (int e = 0; e < 16; ++e) hi[e] = x[e];
            ptx::tmem_ld16(o_mem + 16 + lanes, lo);
            ptx::tmem_ld_wait16(lo);
          } else {
            uint32_t more[4] = {x[8], 0, 0, 0};
            if constexpr (kCols == 8) {
              ptx::tmem_ld4(o_mem + 16 + lanes, more);
              ptx::tmem_ld_wait4(more);
            }
#pragma unroll
            for (int e = 0; e < kCols; ++e) {
              hi[e] = x[e];
              lo[e] = x[kCols + e] - 128u * more[0];
            }
          }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.oempty));
      }
      auto store = [&](int e, int dim, int y) {
        const int at = u.flat0 + e;
        const long long to = (long long)(u.row0 + at / a.group) * f.ldy + (u.head * a.group + at % a.group) * D + dim;
        if (a.y_bytes == 1) ((int8_t*)f.y)[to] = (int8_t)y;
        else ((int*)f.y)[to] = y;
      };
      if (u.team == 1) {
        const Reciprocal mine = reciprocal(max(L, 1ll), V);
#pragma unroll
        for (int e = 0; e < kCols; ++e) {
          if (e < nc) {
            Reciprocal rec;
            rec.rho = __shfl_sync(0xFFFFFFFFu, mine.rho, e);
            rec.a = __shfl_sync(0xFFFFFFFFu, mine.a, e);
            rec.V = __shfl_sync(0xFFFFFFFFu, V, e);
            const bool any = __shfl_sync(0xFFFFFFFFu, (int)(L > 0), e) != 0;
            if (e % kGroups == w && key < D && ok) {
              const int at = (u.head * a.group + (u.flat0 + e) % a.group) * D + key;
              store(e, key, clipped(requantised(any ? quotient((int)hi[e], (int)lo[e], rec) : 0, a.out[at]), a.lo, a.hi));
            }
          }
        }
      } else {
        const int own = owned(D, u.team);
        if (key < D) {
          const uint32_t to = ptx::cluster_addr(osum + (uint32_t)((u.member * own + key % own) * kCols * 8), (uint32_t)(rank - u.member + key / own));
#pragma unroll
          for (int e = 0; e < kCols; ++e) {
            if (e < nc && e % kGroups == w) {
              ptx::st_cluster(to + 8 * e, hi[e]);
              ptx::st_cluster(to + 8 * e + 4, lo[e]);
            }
          }
        }
        const uint32_t peer = (uint32_t)(rank - u.member + min(lane, u.team - 1));
        if (me == 0) {
          const uint32_t to = ptx::cluster_addr(ptx::smem_u32(&sh.team_sum[u.member][0]), peer);
          for (int e = 0; e < nc; ++e) {
            const unsigned long long v = (unsigned long long)__shfl_sync(0xFFFFFFFFu, L, e);
            if (lane < u.team) {
              ptx::st_cluster(to + 8 * e, (uint32_t)v);
              ptx::st_cluster(to + 8 * e + 4, (uint32_t)(v >> 32));
            }
          }
        }
        ptx::named_barrier(1, 32 * kSoft);              // all of this CTA's sums are on their way
        if (me == 0 && lane < u.team) ptx::mbar_arrive_cluster(ptx::cluster_addr(ptx::smem_u32(&sh.sums[u.cls]), peer));
        __syncwarp();
        const int mine = min(tid - 128, own * nc - 1), my_dim = min(u.member * own + mine % own, D - 1);
        const int4 my_out = a.out[(u.head * a.group + (u.flat0 + mine / own) % a.group) * D + my_dim];      // of the first output, asked for early
        ok = ok && team_wait(&sh.sums[u.cls], team_phases >> u.cls & 1);
        team_phases ^= 1u << u.cls;
        for (int i = tid - 128; ok && i < own * nc; i += 32 * kSoft) {
          const int dl = i % own, e = i / own, dim = u.member * own + dl;
          if (dim >= D) continue;
          int hi_all = 0, lo_all = 0;                   // no more than a row's sums
          long long all = 0;
          for (int m = 0; m < u.team; ++m) {
            const int* o = osums + ((m * own + dl) * kCols + e) * 2;
            hi_all += o[0];
            lo_all += o[1];
            all += sh.team_sum[m][e];
          }
          const int at = (u.head * a.group + (u.flat0 + e) % a.group) * D + dim;
          store(e, dim, clipped(requantised(all ? quotient(hi_all, lo_all, reciprocal(all, sh.vtop[e])) : 0, i == tid - 128 ? my_out : a.out[at]), a.lo, a.hi));
        }
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.uempty[ur.slot]));
      ur.next(kUnitsS);
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (warp == 2) ptx::tmem_dealloc(tmem, At::kColumns);
  ptx::cluster_arrive();                                // nobody leaves while another CTA may still write into its memory
  ptx::cluster_wait();
}

template <int D, int kCols, int kGroups>
cudaError_t configure() {
  typedef Shape<kCols, kGroups> At;
  static_assert(sizeof(SharedS<At>) + 4 * (kWeightSegments * 32 + kClasses * (kMaxChunks + 1)) + At::kDynamic + 1024 <= (kGroups == 4 ? 228 : 114) * 1024,
                "shared memory");
  cudaError_t e = cudaFuncSetAttribute(split_kernel<D, kCols, kGroups>, cudaFuncAttributeMaxDynamicSharedMemorySize, At::kDynamic);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(split_kernel<D, kCols, kGroups>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  return e == cudaSuccess ? cudaFuncSetAttribute(split_kernel<D, kCols, kGroups>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) : e;
}

template <int D>
cudaError_t configure() {
  cudaError_t e = configure<D, 4, 4>();
  if (e == cudaSuccess) e = configure<D, 8, 4>();
  if (e == cudaSuccess) e = configure<D, 16, 4>();
  if (e == cudaSuccess) e = configure<D, 4, 2>();
  if (e == cudaSuccess) e = configure<D, 8, 2>();
  return e == cudaSuccess ? configure<D, 16, 2>() : e;
}

template <int kGroups>
cudaLaunchConfig_t config(int cluster, int clusters, cudaLaunchAttribute* attr, cudaStream_t stream) {
  typedef Shape<4, kGroups> At;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(cluster * clusters));
  cfg.blockDim = dim3(At::kThreads);
  cfg.dynamicSmemBytes = At::kDynamic;
  cfg.stream = stream;
  attr->id = cudaLaunchAttributeClusterDimension;
  attr->val.clusterDim.x = (unsigned)cluster;
  attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cfg;
}

template <int D, int kCols>
cudaError_t launch(const AttnArgs& a, const CacheArgs& c, const ForwardArgs& f, const CUtensorMap& k_map, const CUtensorMap& v_map,
                   cudaStream_t stream) {
  // at most: whole units and one that is not for each request, or the units of each token by itself
  const long long units = std::min((long long)f.rows * a.group / kCols + f.n, (long long)f.rows * ((a.group + kCols - 1) / kCols)) * a.kv;
  SplitArgs s;
  s.chunks = (f.n + 31) / 32;
  s.cluster = kLeastCluster;
  s.one_team = 0;
  const bool pairs = units > a.sms;                     // their sums have no room for a team of more than eight
  for (int n = std::min(kMaxTeam, f.width); n > kLeastCluster && !s.one_team && !pairs; --n) {
    if (a.clusters[n] < units) continue;
    s.cluster = n;
    s.one_team = 1;
  }
  // (of CTAs of which two fit an SM the occupancy query, too, counts one: 64 requests take 43 us with as many clusters, 35 with twice as many)
  const int most = std::max(1, a.clusters[s.cluster]) * (pairs ? 2 : 1);
  // Blocks of a request that are still left to one CTA: such that the longest contexts' teams fill the GPU, and 16 at most, since contexts may
  // differ (64 requests with up to 64 blocks, 512 units: 47.7, 39.5, 35.1, 35.6 us with 2, 4, 8, 16).
  int team = 1;
  while (2 * team <= s.cluster && 2 * team * units <= (long long)most * s.cluster) team *= 2;
  s.per_cta = std::min(16, (f.width + team - 1) / team);
  const int clusters = (int)std::min<long long>(most, units);
  cudaLaunchAttribute attr;
  if (pairs) {
    const cudaLaunchConfig_t cfg = config<2>(s.cluster, clusters, &attr, stream);
    return cudaLaunchKernelEx(&cfg, split_kernel<D, kCols, 2>, k_map, v_map, a, c, f, s);
  }
  const cudaLaunchConfig_t cfg = config<4>(s.cluster, clusters, &attr, stream);
  return cudaLaunchKernelEx(&cfg, split_kernel<D, kCols, 4>, k_map, v_map, a, c, f, s);
}

template <int D>
cudaError_t launch(const AttnArgs& a, const CacheArgs& c, const ForwardArgs& f, const CUtensorMap& k_map, const CUtensorMap& v_map,
                   cudaStream_t stream) {
  const int cols = attn_split_cols(a, f);
  return cols == 4 ? launch<D, 4>(a, c, f, k_map, v_map, stream)
                   : cols == 8 ? launch<D, 8>(a, c, f, k_map, v_map, stream) : launch<D, 16>(a, c, f, k_map, v_map, stream);
}

}  // namespace

int attn_split_cols(const AttnArgs& a, const ForwardArgs& f) {
  const long long flat = ((long long)f.rows * a.group + f.n - 1) / f.n;                   // rows of a request, about
  return flat <= 4 ? 4 : flat <= 8 ? 8 : 16;
}

cudaError_t configure_attn_split(AttnArgs* a) {
  cudaError_t e = configure<32>();
  if (e == cudaSuccess) e = configure<64>();
  if (e == cudaSuccess) e = configure<128>();
  for (int i = kLeastCluster; i <= kMaxTeam && e == cudaSuccess; ++i) {
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = config<4>(i, 1, &attr, nullptr);
    e = cudaOccupancyMaxActiveClusters(a->clusters + i, split_kernel<128, 4, 4>, &cfg);
  }
  return e;
}

cudaError_t launch_attn_split(const AttnArgs& a, const CacheArgs& c, const ForwardArgs& f, const CUtensorMap& k_map, const CUtensorMap& v_map,
                              cudaStream_t stream) {
  return a.dim == 128 ? launch<128>(a, c, f, k_map, v_map, stream)
                      : a.dim == 64 ? launch<64>(a, c, f, k_map, v_map, stream) : launch<32>(a, c, f, k_map, v_map, stream);
}

}  // namespace iodf
