// Projection with low-rank adapters of many requests (include/iodf.h: iodf_proj_forward).
//
// Two kernels. The first finds the adapter of every row and computes h, the 8-bit rank channels; the second multiplies
//   D[128 output channels][rows of a tile] = W x^T + up h^T     (tcgen05 kind::i8, int32 sums in tensor memory)
// and requantises. The output channels are the MMA's M, so a thread of the epilogue owns one channel and keeps its
// constants in registers. An adapter is one more step along K with its own operands: `up`, and h with
// zeros in the rows of other adapters, so a tile may mix any number of them in one accumulator. The second kernel is
// launched while the first runs (programmatic dependent launch) and waits for it only where it needs h.
#include "proj_kernel.h"

#include <cuda.h>

#include <limits.h>

#include <algorithm>

#include "../../include/iodf.h"
#include "iodf_dev.h"
#include "ptx_cluster.cuh"

namespace iodf {
namespace {

constexpr int kEpiWarps = 16;
constexpr int kFill = 128;
constexpr int kMainThreads = 256 + 32 * kEpiWarps;   // warp 0 copies, 1 MMAs, 2 tensor memory, 4-7 adapter steps, 8-23 epilogue
constexpr int kMaxRing = 6;
constexpr int kBytesW = kProjTileN * kProjStage;
constexpr int kDownRows = kProjDownRows;
constexpr int kDownRing = 6;             // stages at most
constexpr int kDownEpiWarps = 8;
constexpr int kDownThreads = 128 + 32 * kDownEpiWarps;   // warp 0 copies, 1 MMAs, 2 tensor memory, 4-11 epilogue
constexpr int kDownStageBytes = kDownRows * kProjStage + kBytesW;
// Up to here a tile (or row) reads every request, above it halves for each row. Read and halved, us: 512 requests 35.5 and 36.7
// (2048 rows, 2048 -> 2048), 30.9 and 31.5 (32768, 512 -> 512), 224 and 240 (16384, 4096 -> 4096); 1024: 38.6 and 39.3, 44.3
// and 43.5, 308 and 310; 2000: 46.6 and 44.5, 73.7 and 70.3, 335 and 341.
constexpr int kScanRequests = 1024;
constexpr int kSlotBits = 20;            // row_slot: an adapter's slot and above it its rank, -1 none, -2 in no request

// D = s32; A int8 (weights), B int8 or uint8, both K-major, M = m, N = n
__device__ __forceinline__ uint32_t idesc(uint32_t n, bool b_unsigned, uint32_t m = 128u) {
  return (2u << 4) | (1u << 7) | ((b_unsigned ? 0u : 1u) << 10) | ((n >> 3) << 17) | ((m >> 4) << 24);
}
// operand words: core matrices 128 bytes apart along K, groups of eight rows sbo apart
__device__ __forceinline__ uint32_t core_lo(uint32_t saddr) { return ptx::umma_desc_lo(saddr, 128u); }
__device__ __forceinline__ uint32_t core_hi(uint32_t sbo) { return (sbo >> 4) | (1u << 14); }
constexpr uint32_t kSwizzledHi = (1024u >> 4) | (1u << 14) | (2u << 29);   // rows of 128 bytes, 128-byte swizzle

// Slot and phase of a ring of barriers, counted (a modulus costs some 70 ns).
struct Turn {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int size) {
    if (++slot == size) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

// Waits until the MMAs have given every slot of a ring back. Nobody else waits for the last of these arrivals, and one that came after
// the CTA had left (or, of a pair, the other CTA's) would find another CTA's shared memory. turn: of the copy that would be next.
__device__ __forceinline__ bool given_back(volatile uint32_t* abort_flag, uint32_t* status, uint64_t* empty, Turn turn, int size) {
  for (int i = 0; i < size; ++i, turn.next(size))
    if (!ptx::quick_wait(abort_flag, status, &empty[turn.slot], turn.phase ^ 1, kSpinLimit)) return false;
  return true;
}

template <bool kPair>
__device__ __forceinline__ void mma(uint32_t d, uint32_t alo, uint32_t ahi, uint32_t blo, uint32_t bhi, uint32_t id, uint32_t acc) {
  if (kPair) ptx::umma_i8_hl_pair(d, alo, ahi, blo, bhi, id, acc);
  else ptx::umma_i8_hl(d, alo, ahi, blo, bhi, id, acc);
}

// The MMAs of a stage: up to four steps of 32 channels, both operands K-major (x with the 128-byte swizzle).
template <bool kPair = false>
__device__ __forceinline__ void stage_mmas(uint32_t d, uint32_t alo, uint32_t blo, uint32_t id, int steps, bool first) {
  mma<kPair>(d, alo, core_hi(1024u), blo, kSwizzledHi, id, first ? 0u : 1u);
  if (steps == 4) {
#pragma unroll
    for (int k = 1; k < 4; ++k) mma<kPair>(d, alo + k * 16, core_hi(1024u), blo + k * 2, kSwizzledHi, id, 1u);
  } else {
    for (int k = 1; k < steps; ++k) mma<kPair>(d, alo + k * 16, core_hi(1024u), blo + k * 2, kSwizzledHi, id, 1u);
  }
}

template <bool kUnsigned>
__device__ __forceinline__ int dot4(int w, int x, int acc) {
  if (kUnsigned) asm("dp4a.s32.u32 %0, %1, %2, %3;" : "=r"(acc) : "r"(w), "r"(x), "r"(acc));
  else asm("dp4a.s32.s32 %0, %1, %2, %3;" : "=r"(acc) : "r"(w), "r"(x), "r"(acc));
  return acc;
}
template <bool kUnsigned>
__device__ __forceinline__ int dot16(int4 w, int4 x, int acc) {
  acc = dot4<kUnsigned>(w.x, x.x, acc);
  acc = dot4<kUnsigned>(w.y, x.y, acc);
  acc = dot4<kUnsigned>(w.z, x.z, acc);
  return dot4<kUnsigned>(w.w, x.w, acc);
}

// 16 bytes of a row of x from channel k0 on; channels beyond the last are zero and not read
__device__ __forceinline__ int4 load_x16(const uint8_t* row, int k0, int K) {
  if (k0 + 16 <= K) return *reinterpret_cast<const int4*>(row + k0);
  int w[4] = {0, 0, 0, 0};
  for (int i = 0; k0 + i < K && i < 16; ++i) w[i >> 2] |= (int)row[k0 + i] << (8 * (i & 3));
  return make_int4(w[0], w[1], w[2], w[3]);
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
  return s >= 0 && s < a.max_adapters ? s : -1;
}

__device__ __forceinline__ int slot_only(int slot_rank) { return slot_rank < 0 ? slot_rank : slot_rank & ((1 << kSlotBits) - 1); }

__device__ __forceinline__ void look_over_request(const ProjArgs& a, int q) {
  const int s0 = a.seg_start[q], s1 = a.seg_start[q + 1], ad = a.seg_adapter[q];
  if (s0 < 0 || s1 < s0 || s1 > a.rows || ad < -1 || ad >= a.max_adapters) atomicAdd(a.status + 1, 1u);
}
// by one warp
__device__ __forceinline__ void look_over_requests(const ProjArgs& a) {
  for (int q = threadIdx.x & 31; q < a.n_seg; q += 32) look_over_request(a, q);
}

__device__ __forceinline__ int8_t rank_value(int acc, int2 q) {
  const int v = (int)(((long long)acc * q.x + (1ll << (30 + q.y))) >> (31 + q.y));
  return (int8_t)min(max(v, -128), 127);
}

// h of 16 rows for one rank channel of adapter `slot`, in the rows that use it. slots: 16-byte aligned, shared memory.
__device__ __forceinline__ void store_rank(int8_t* h, int rp, const uint32_t (&v)[16], int2 q, int slot, const int* slots) {
  int s[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int4 t = reinterpret_cast<const int4*>(slots)[i];
    s[4 * i] = t.x; s[4 * i + 1] = t.y; s[4 * i + 2] = t.z; s[4 * i + 3] = t.w;
  }
  const long long round = 1ll << (30 + q.y);
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int o = min(max((int)(((long long)(int)v[e] * q.x + round) >> (31 + q.y)), -128), 127);
    if (s[e] == slot) h[e * rp] = (int8_t)o;
  }
}

// Is row r the first of its tile with adapter slots[r]? `starts` has a bit for each row whose slot differs from the row's above:
// only those are looked at (a walk over all rows above took 4000 clocks where a request starts low in a tile).
__device__ __forceinline__ bool first_of_slot(const int* slots, const uint32_t* starts, int r) {
  const int s = slots[r];
  if (s < 0 || !(starts[r >> 5] >> (r & 31) & 1)) return false;
  for (int w = 0; w <= r >> 5; ++w)
    for (uint32_t b = w < r >> 5 ? starts[w] : starts[w] & ((1u << (r & 31)) - 1); b; b &= b - 1)
      if (slots[w * 32 + __ffs((int)b) - 1] == s) return false;
  return true;
}

// ---- h for few rows: a block per row and eight rank channels, a quarter of K per warp ----------------------
// A chain of dependent loads bounds it (request, rank, adapter and x). One row, 1024 -> 4096: 4.8 us without adapters, 5.8 with one of
// rank 16. Beyond that a block adds about 0.35 ns and 0.68 ps for each channel of K (the fit that down_rows_ns uses).
template <bool kUnsigned>
__global__ void __launch_bounds__(128) down_rows_kernel(const ProjArgs a) {
  __shared__ int part[4][8], found;
  ptx::grid_launch_dependents();
  const int row = blockIdx.x, g = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int slot;
  if (a.n_seg <= kScanRequests) {                       // all requests at once: one trip to memory instead of one per halving
    if (threadIdx.x == 0) found = -2;
    __syncthreads();
    for (int q = threadIdx.x; q < a.n_seg; q += blockDim.x) {
      const int s0 = a.seg_start[q], s1 = a.seg_start[q + 1], ad = a.seg_adapter[q];
      if (s0 <= row && row < s1) found = ad >= 0 && ad < a.max_adapters ? ad : -1;
    }
    __syncthreads();
    slot = found;
  } else {
    slot = slot_of_row(a, row);
  }
  if (row == 0 && g == gridDim.y - 1 && warp == 3) look_over_requests(a);      // a block whose rank channels are mostly padding
  const int rank = slot < 0 ? 0 : a.rank[slot];
  if (g == 0 && threadIdx.x == 0) a.row_slot[row] = slot < 0 ? slot : slot | rank << kSlotBits;
  if (g * 8 >= rank) return;
  // 32 lanes: four chunks of 16 channels x eight rank channels, 512 contiguous bytes of `down`
  const int chunk = lane >> 3, j = lane & 7;
  const uint8_t* d = a.down + ((size_t)slot * a.stages * a.rp + g * 8) * kProjStage + j * 16;
  const uint8_t* x = a.x + (size_t)row * a.ldx;
  int acc = 0;
#pragma unroll 4
  for (int c = warp * 4 + chunk; c * 16 < a.k; c += 16)
    acc = dot16<kUnsigned>(*reinterpret_cast<const int4*>(d + (size_t)(c >> 3) * a.rp * kProjStage + (c & 7) * 128), load_x16(x, c * 16, a.k), acc);
  acc += __shfl_xor_sync(0xFFFFFFFFu, acc, 8);
  acc += __shfl_xor_sync(0xFFFFFFFFu, acc, 16);
  if (lane < 8) part[warp][lane] = acc;
  __syncthreads();
  if (threadIdx.x < 8) {
    acc = part[0][threadIdx.x] + part[1][threadIdx.x] + part[2][threadIdx.x] + part[3][threadIdx.x];
    a.h[(size_t)row * a.rp + g * 8 + threadIdx.x] = rank_value(acc, a.down_rq[slot * a.rp + g * 8 + threadIdx.x]);
  }
}

// ---- h for many rows: the same product as the main kernel's, M = the rank channels of 128 / rp adapters --------
// Tiles of 128 rows; each reads x once per group of 128 / rp adapters that its rows use (mostly one group). A block's time is
// mostly latency (requests, x, sums, h), so up to three blocks share an SM when there are more tiles than SMs. 16384 x 4096, rank 64:
// some 15 us of the call's 185.
struct DownShared {
  uint64_t full[kDownRing], empty[kDownRing], dfull, dempty;
  uint32_t abort_flag, tmem;
  int n_slots;
  uint32_t starts[kDownRows / 32];
  alignas(16) int slot[kDownRows];
  int list[kDownRows];
};

__global__ void __launch_bounds__(kDownThreads) down_tile_kernel(const __grid_constant__ CUtensorMap xmap, const ProjArgs a, const int ring) {
  extern __shared__ uint8_t raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  __shared__ DownShared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row0 = blockIdx.x * kDownRows, per = kProjTileN / a.rp;      // adapters per MMA
  if (tid == 0) {
    for (int i = 0; i < ring; ++i) {
      ptx::mbar_init(ptx::smem_u32(&sh.full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.empty[i]), 1);
    }
    ptx::mbar_init(ptx::smem_u32(&sh.dfull), 1);
    ptx::mbar_init(ptx::smem_u32(&sh.dempty), kDownEpiWarps);
    ptx::mbar_init_fence();
    sh.abort_flag = 0;
    sh.n_slots = 0;
  }
  if (warp == 2) ptx::tmem_alloc(ptx::smem_u32(&sh.tmem), (uint32_t)kDownRows);
  const bool scan = a.n_seg <= kScanRequests;
  if (tid < kDownRows) sh.slot[tid] = scan || row0 + tid >= a.rows ? -2 : slot_of_row(a, row0 + tid);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  // Only now: a block of the main kernel on this SM could otherwise take the tensor memory first and wait for this kernel.
  ptx::grid_launch_dependents();
  if (scan) {                                         // each request writes its rows of the tile: one trip to memory
    for (int q = tid; q < a.n_seg; q += kDownThreads) {
      const int s0 = a.seg_start[q], s1 = a.seg_start[q + 1], ad = a.seg_adapter[q];
      const int lo = max(s0, row0), hi = min(min(s1, row0 + kDownRows), a.rows);
      if (lo >= hi) continue;
      const int s = ad >= 0 && ad < a.max_adapters ? ad : -1;
      for (int r = lo; r < hi; ++r) sh.slot[r - row0] = s;
    }
    __syncthreads();
  }
  if (tid < kDownRows) {
    const int s = sh.slot[tid];
    if (row0 + tid < a.rows) a.row_slot[row0 + tid] = s;
    const uint32_t starts = __ballot_sync(0xFFFFFFFFu, tid == 0 || sh.slot[tid - 1] != s);
    if (lane == 0) sh.starts[warp] = starts;
  }
  __syncthreads();                                    // the adapters of the tile, each once, in any order
  if (tid < kDownRows && first_of_slot(sh.slot, sh.starts, tid)) sh.list[atomicAdd(&sh.n_slots, 1)] = sh.slot[tid];
  __syncthreads();
  const int n_slots = sh.n_slots, groups = (n_slots + per - 1) / per;
  const uint32_t base = ptx::smem_u32(smem), tmem = sh.tmem;
  volatile uint32_t* abort_flag = &sh.abort_flag;

  if (warp == 0 && ptx::elect_one()) {
    Turn turn;
    for (int g = 0; g < groups; ++g) {
      const int n = min(per, n_slots - g * per);
      for (int ks = 0; ks < a.stages; ++ks, turn.next(ring)) {
        const int s = turn.slot;
        if (!ptx::quick_wait(abort_flag, a.status, &sh.empty[s], turn.phase ^ 1, kSpinLimit)) { g = groups; break; }
        const uint32_t st = base + s * kDownStageBytes, bar = ptx::smem_u32(&sh.full[s]);
        ptx::mbar_expect_tx(bar, (uint32_t)(kDownRows * kProjStage + n * a.rp * kProjStage));
        ptx::tile_g2s(st, &xmap, ks * kProjStage, row0, bar);
        for (int i = 0; i < n; ++i)
          ptx::bulk_g2s(st + kDownRows * kProjStage + i * a.rp * kProjStage,
                        a.down + ((size_t)sh.list[g * per + i] * a.stages + ks) * a.rp * kProjStage, (uint32_t)(a.rp * kProjStage), bar);
      }
    }
    given_back(abort_flag, a.status, sh.empty, turn, ring);
  } else if (warp == 1 && ptx::elect_one()) {
    const uint32_t id = idesc(kDownRows, a.x_unsigned);
    Turn turn;
    for (int g = 0; g < groups; ++g) {
      if (!ptx::quick_wait(abort_flag, a.status, &sh.dempty, (g & 1) ^ 1, kSpinLimit)) break;
      ptx::tc_fence_after();
      for (int ks = 0; ks < a.stages; ++ks, turn.next(ring)) {
        const int s = turn.slot;
        if (!ptx::quick_wait(abort_flag, a.status, &sh.full[s], turn.phase, kSpinLimit)) { g = groups; break; }
        ptx::tc_fence_after();
        const uint32_t st = base + s * kDownStageBytes;
        stage_mmas(tmem, core_lo(st + kDownRows * kProjStage), ptx::umma_desc_lo(st, 16u), id, min(4, (a.k - ks * kProjStage + 31) >> 5), ks == 0);
        ptx::umma_commit(ptx::smem_u32(&sh.empty[s]));
      }
      ptx::umma_commit(ptx::smem_u32(&sh.dfull));
    }
  } else if (warp == 3 && blockIdx.x == 0) {
    look_over_requests(a);
  } else if (warp >= 4) {
    const int q = warp & 3, half = (warp - 4) >> 2, m = q * 32 + lane, j = m % a.rp;
    for (int g = 0; g < groups; ++g) {
      const int i = g * per + m / a.rp;
      const int slot = i < n_slots ? sh.list[i] : -3;
      const bool used = slot >= 0;
      const int2 rq = used ? a.down_rq[slot * a.rp + j] : make_int2(1 << 30, 0);
      if (!__all_sync(0xFFFFFFFFu, ptx::quick_wait(abort_flag, a.status, &sh.dfull, g & 1, kSpinLimit))) break;
      ptx::tc_fence_after();
      if (__any_sync(0xFFFFFFFFu, used)) {
        for (int c = half * (kDownRows / 2); c < (half + 1) * (kDownRows / 2); c += 16) {
          uint32_t v[16];
          ptx::tmem_ld16(tmem + ((uint32_t)(q * 32) << 16) + c, v);
          ptx::tmem_ld_wait16(v);
          store_rank(a.h + (size_t)(row0 + c) * a.rp + j, a.rp, v, rq, slot, sh.slot + c);
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.dempty));
    }
  }
  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 2) ptx::tmem_dealloc(tmem, (uint32_t)kDownRows);
}

// ---- the projection ----------------------------------------------------------------------------------------------
// Persistent: units of one row tile and some output tiles; each output tile is an item: a product over K into one of two
// accumulators, the steps of its rows' adapters, the epilogue. Two forms, by whether an x tile fits in shared memory:
//   fused  (K up to about 1000) a CTA per unit of `chunk` output tiles. It holds the unit's x tile, read once for all
//          items, and computes h itself, as further items in front of the output tiles: the sums of `down x^T` go through the
//          same accumulators, and h through global memory to the warps that lay it out. That repeats the product for
//          every unit of a row tile and saves a launch and a wait for it.
//   paired (larger K) two CTAs per unit of two output tiles, one each, and one MMA over both (M = 256). Each reads half of
//          the x tile: a stage is 32 KB of copies and 32 KB of operand reads per SM for 512 clocks of MMAs, where single CTAs
//          have 48 KB of each, more than the 128 bytes per clock of shared memory. down_tile_kernel computes h before.
// 65536 x 512 -> 512, uint8, rank 32 (fused): 34.7 us, 1.1 POP/s, tensor pipe 27 % active. Of the 72 000 clocks of a CTA with two units
// (108 of 148 have two, 40 one; clock stamps) the epilogue of its eight output tiles takes 34 000 (some 1760 per 32 rows: 300 load, 720
// requantisation, 280 transposition, 460 stores). The rest is the chain in front of a unit's first output tile (20 000 before the
// first unit: start, requests, copies of `down`, the product, h and its way through L2; 8 000 before the second, as there is room for one
// x tile only) and 8 000 of waits between tiles. 32768 x 256 -> 256: 14.3 us, one unit: 17 000 of 27 000 clocks before its first
// output tile. 16384 x 4096 -> 4096, rank 64 (paired): 171 of the call's 185 us, tensor pipe 85 % active.
constexpr int kMaxTile = 256;

constexpr int kMaxX = 16;

struct MainShared {
  uint64_t xfull[kMaxX], xempty[kMaxX], wfull[kMaxRing], wempty[kMaxRing], apeer[2], afull[2], aempty[2], tfull[2], tempty[2], lready[2], lfree[2], hready;
  uint32_t abort_flag, tmem;
  int message[2];                        // an adapter step: its adapters, 256: the tile's last
  int n_list[2];
  uint32_t starts[kMaxTile / 32], firsts[kMaxTile / 32];      // rows with another adapter than the row above, than any row above: a bit each
  alignas(16) int slot[2][kMaxTile];     // of a unit: adapter of each row
  int list[2][kMaxTile];                 //            every adapter once
  uint32_t live[2][kMaxTile / 32];       // of a unit: the rows that some request owns
  alignas(16) uint32_t out[kEpiWarps][256];
};

struct MainShape {
  int tile;                              // rows per tile: 128 or 256
  int xring, wring;                      // stages of x and of weights in shared memory
  int tmem_cols;
  int chunk, chunks;                     // output tiles of a unit (paired: of each CTA), units of a row tile
  int units;
  int abytes;                            // an adapter step's operands: `up`, h
  int step_adapters;                     // adapters of a step
  int vector_y;                          // 8-bit rows of y lie on 4-byte boundaries
  int clip;                              // the clip is narrower than the output's type
};

// (acc M0 + addend) >> (31 + s): the high word of a multiply-add, shifted; s = 0 (shift is 0 then too) needs one bit below it
template <bool kAnyShift>
__device__ __forceinline__ int requantised(int acc, int4 rq, long long add, int shift) {
  const long long p = (long long)acc * rq.x + add;
  const int o = (int)(p >> 32) >> shift;
  return kAnyShift && rq.y == 0 ? (int)(p >> 31) : o;
}

// {sat(y3), sat(y2), sat(y1), sat(y0)}, y0 in the lowest byte
template <class YT>
__device__ __forceinline__ uint32_t pack4(int y0, int y1, int y2, int y3) {
  uint32_t t, w;
  if (YT(-1) < YT(0)) {
    asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(t) : "r"(y3), "r"(y2), "r"(0));
    asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(w) : "r"(y1), "r"(y0), "r"(t));
  } else {
    asm("cvt.pack.sat.u8.s32.b32 %0, %1, %2, %3;" : "=r"(t) : "r"(y3), "r"(y2), "r"(0));
    asm("cvt.pack.sat.u8.s32.b32 %0, %1, %2, %3;" : "=r"(w) : "r"(y1), "r"(y0), "r"(t));
  }
  return w;
}

// Four words of four rows, one word per channel -> four words of four channels, one per row.
__device__ __forceinline__ void transpose4(int4 t, uint32_t* w) {
  const uint32_t ab = __byte_perm(t.x, t.y, 0x5140), cd = __byte_perm(t.z, t.w, 0x5140);    // rows 0 and 1 of channels 0, 1 and 2, 3
  const uint32_t ef = __byte_perm(t.x, t.y, 0x7362), gh = __byte_perm(t.z, t.w, 0x7362);
  w[0] = __byte_perm(ab, cd, 0x5410);
  w[1] = __byte_perm(ab, cd, 0x7632);
  w[2] = __byte_perm(ef, gh, 0x5410);
  w[3] = __byte_perm(ef, gh, 0x7632);
}

// true if it is for all 128 threads of warps 4-7 (and a barrier of theirs)
__device__ __forceinline__ bool fill_all(bool fine) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
      "barrier.cta.red.and.pred p, 1, 128, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)fine)
      : "memory");
  return r != 0;
}

template <class YT, bool kAnyShift, bool kFused>
__global__ void __launch_bounds__(kMainThreads, 1) proj_tile_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap, const ProjArgs a, const MainShape shp) {
  extern __shared__ uint8_t raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  __shared__ MainShared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr bool kPair = !kFused;
  const int RT = shp.tile, half = kPair ? RT / 2 : RT;      // rows of x (and of h) in this CTA's shared memory
  const int part = kPair ? (int)ptx::cluster_rank() : 0;
  const int unit0 = kPair ? blockIdx.x / 2 : blockIdx.x, unit_step = kPair ? gridDim.x / 2 : gridDim.x;
  const uint32_t xbytes = (uint32_t)(half * kProjStage);
  if (tid == 0) {
    for (int i = 0; i < shp.xring; ++i) {
      ptx::mbar_init(ptx::smem_u32(&sh.xfull[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.xempty[i]), 1);
    }
    for (int i = 0; i < shp.wring; ++i) {
      ptx::mbar_init(ptx::smem_u32(&sh.wfull[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.wempty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(ptx::smem_u32(&sh.afull[i]), kFill + 1);
      ptx::mbar_init(ptx::smem_u32(&sh.aempty[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.apeer[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.tfull[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.tempty[i]), kPair ? 2 * kEpiWarps : kEpiWarps);
      ptx::mbar_init(ptx::smem_u32(&sh.lready[i]), kFill);
      ptx::mbar_init(ptx::smem_u32(&sh.lfree[i]), kEpiWarps);
    }
    ptx::mbar_init(ptx::smem_u32(&sh.hready), kEpiWarps);
    ptx::mbar_init_fence();
    sh.abort_flag = 0;
  }
  if (kPair) {                                          // both CTAs' barriers are there before either arrives on the other's
    ptx::cluster_arrive();
    ptx::cluster_wait();
  }
  if (warp == 2) {
    if (kPair) ptx::tmem_alloc_pair(ptx::smem_u32(&sh.tmem), (uint32_t)shp.tmem_cols);
    else ptx::tmem_alloc(ptx::smem_u32(&sh.tmem), (uint32_t)shp.tmem_cols);
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t base = ptx::smem_u32(smem), wbase = base + shp.xring * xbytes, abase = wbase + shp.wring * kBytesW, tmem = sh.tmem;
  volatile uint32_t* abort_flag = &sh.abort_flag;
  auto wait = [&](uint64_t* bar, uint32_t parity) { return ptx::quick_wait(abort_flag, a.status, bar, parity, kSpinLimit); };
  const int per = kProjTileN / a.rp;                  // adapters of one product `down x^T`
  const bool adapters = a.n_seg != 0;

  // the output tiles of unit u: fused, first_tile to last_tile - 1 in turn; paired, one (the second CTA's may lie behind the last)
  auto first_tile = [&](int u) { return kPair ? u % shp.chunks * 2 + part : u % shp.chunks * shp.chunk; };
  auto last_tile = [&](int u) { return kPair ? first_tile(u) + 1 : min(first_tile(u) + shp.chunk, a.tiles_n); };
  auto stored_tile = [&](int tn) { return kPair ? min(tn, a.tiles_n - 1) : tn; };      // whose weights stand in for one behind the last
  // x of a fused unit: xring is once or twice the stages, unit ui has slots from xslot0(ui) on. Paired: a stage's x and
  // weights are slots of one ring with one barrier, the first CTA's.
  const int sets = kPair ? 1 : shp.xring / a.stages;
  auto xslot0 = [&](int ui) { return sets == 2 ? (ui & 1) * a.stages : 0; };
  auto xphase = [&](int ui) { return (uint32_t)(sets == 2 ? ui >> 1 : ui) & 1u; };

  if (!kPair && warp == 3 && ptx::elect_one()) {
    int ui = 0;
    bool ok = true;
    for (int u = unit0; ok && u < shp.units; u += unit_step, ++ui)
      for (int ks = 0; ks < a.stages; ++ks) {
        const int s = xslot0(ui) + ks;
        if (!(ok = wait(&sh.xempty[s], xphase(ui) ^ 1))) break;
        const uint32_t bar = ptx::smem_u32(&sh.xfull[s]);
        ptx::mbar_expect_tx(bar, xbytes);
        ptx::tile_g2s(base + s * xbytes, &xmap, ks * kProjStage, u / shp.chunks * RT, bar);
      }
    for (int i = 0; i < sets; ++i)                      // as given_back
      for (int ks = 0; ok && ks < a.stages; ++ks) ok = wait(&sh.xempty[xslot0(ui + i) + ks], xphase(ui + i) ^ 1);
  } else if (warp == 0 && ptx::elect_one()) {
    Turn turn;
    int ui = 0;
    bool ok = true;
    for (int u = unit0; ok && u < shp.units; u += unit_step, ++ui) {
      const int t0 = first_tile(u), t1 = last_tile(u);
      if (kFused && adapters) {
        if (!(ok = wait(&sh.lready[ui & 1], (ui >> 1) & 1))) break;
        const int n_list = sh.n_list[ui & 1];
        for (int g = 0; ok && g < n_list; g += per) {
          const int n = min(per, n_list - g), parts = per / n * n;     // fewer adapters: copies, see the epilogue
          for (int ks = 0; ks < a.stages; ++ks, turn.next(shp.wring)) {
            if (!(ok = wait(&sh.wempty[turn.slot], turn.phase ^ 1))) break;
            const uint32_t bar = ptx::smem_u32(&sh.wfull[turn.slot]), dst = wbase + turn.slot * kBytesW;
            ptx::mbar_expect_tx(bar, (uint32_t)(parts * a.rp * kProjStage));
            for (int i = 0; i < parts; ++i)
              ptx::bulk_g2s(dst + i * a.rp * kProjStage, a.down + ((size_t)sh.list[ui & 1][g + i % n] * a.stages + ks) * a.rp * kProjStage,
                            (uint32_t)(a.rp * kProjStage), bar);
          }
        }
      }
      for (int tn = t0; ok && tn < t1; ++tn)
        for (int ks = 0; ks < a.stages; ++ks, turn.next(shp.wring)) {
          if (!(ok = wait(&sh.wempty[turn.slot], turn.phase ^ 1))) break;
          const uint32_t bar = ptx::smem_u32(&sh.wfull[turn.slot]);
          if (kPair) {                                  // both CTAs' copies count on the first one's barrier
            if (part == 0) ptx::mbar_expect_tx(bar, 2u * (kBytesW + xbytes));
            const uint32_t to = ptx::cluster_addr(bar, 0u);
            ptx::tile_g2s_pair(base + turn.slot * xbytes, &xmap, ks * kProjStage, u / shp.chunks * RT + part * half, to);
            ptx::tile_g2s_pair(wbase + turn.slot * kBytesW, &wmap, 0, (stored_tile(tn) * a.stages + ks) * kProjTileN, to);
          } else {
            ptx::mbar_expect_tx(bar, kBytesW);
            ptx::bulk_g2s(wbase + turn.slot * kBytesW, a.w + ((size_t)tn * a.stages + ks) * kBytesW, kBytesW, bar);
          }
        }
    }
    if (ok) given_back(abort_flag, a.status, sh.wempty, turn, shp.wring);
  } else if (warp == 1 && part == 1 && ptx::elect_one()) {
    // the second CTA of a pair tells the first, which issues the MMAs, that its half of an adapter step is laid out
    int ai = 0;
    bool ok = true;
    for (int u = unit0; adapters && ok && u < shp.units; u += unit_step)
      for (int last = 0; ok && !last; ++ai) {
        if (!(ok = wait(&sh.afull[ai & 1], (ai >> 1) & 1))) break;
        last = sh.message[ai & 1] & 256;
        ptx::mbar_arrive_cluster(ptx::cluster_addr(ptx::smem_u32(&sh.apeer[ai & 1]), 0u));
      }
  } else if (warp == 1 && part == 0 && ptx::elect_one()) {
    const uint32_t m_rows = kPair ? 256u : 128u;
    const uint32_t id = idesc((uint32_t)RT, a.x_unsigned, m_rows), ida = idesc((uint32_t)RT, false, m_rows);
    const uint32_t hhi = core_hi(128u);
    Turn wturn;
    int ai = 0, ti = 0, ui = 0;
    bool ok = true;
    auto commit = [&](uint64_t* bar) {
      if (kPair) ptx::umma_commit_pair(ptx::smem_u32(bar));
      else ptx::umma_commit(ptx::smem_u32(bar));
    };
    auto wait_peer = [&](uint64_t* bar, uint32_t parity) {      // what the other CTA released into the barrier, acquired at cluster scope
      if (!wait(bar, parity)) return false;
      if (kPair) ptx::mbar_acquire_cluster(ptx::smem_u32(bar), parity);
      return true;
    };
    auto product = [&](bool first, bool last) {         // one accumulator: all stages of K; the unit's first and last item
      ok = wait_peer(&sh.tempty[ti & 1], ((ti >> 1) & 1) ^ 1);
      if (!ok) return;
      ptx::tc_fence_after();
      const uint32_t d = tmem + (ti & 1) * RT;
      for (int ks = 0; ks < a.stages; ++ks, wturn.next(shp.wring)) {
        const int ws = wturn.slot, xs = kPair ? ws : xslot0(ui) + ks;
        if (!kPair && first && !(ok = wait(&sh.xfull[xs], xphase(ui)))) return;
        if (!(ok = wait(&sh.wfull[ws], wturn.phase))) return;
        ptx::tc_fence_after();
        stage_mmas<kPair>(d, core_lo(wbase + ws * kBytesW), ptx::umma_desc_lo(base + xs * xbytes, 16u), id, min(4, (a.k - ks * kProjStage + 31) >> 5), ks == 0);
        commit(&sh.wempty[ws]);
        if (!kPair && last) commit(&sh.xempty[xs]);
      }
    };
    for (int u = unit0; ok && u < shp.units; u += unit_step, ++ui) {
      const int t0 = first_tile(u), t1 = last_tile(u);
      bool first = true;                                // no item of the unit has waited for its x yet
      if (kFused && adapters) {
        if (!(ok = wait(&sh.lready[ui & 1], (ui >> 1) & 1))) break;
        const int n_list = sh.n_list[ui & 1];
        first = n_list == 0;
        for (int g = 0; ok && g < n_list; g += per, ++ti) {
          product(g == 0, false);
          if (ok) commit(&sh.tfull[ti & 1]);
        }
      }
      for (int tn = t0; ok && tn < t1; ++tn, ++ti) {
        product(first && tn == t0, tn + 1 == t1);
        const uint32_t d = tmem + (ti & 1) * RT;
        for (int last = !adapters; ok && !last; ++ai) {
          if (!(ok = wait(&sh.afull[ai & 1], (ai >> 1) & 1))) break;
          if (kPair && !(ok = wait_peer(&sh.apeer[ai & 1], (ai >> 1) & 1))) break;
          ptx::tc_fence_after();
          const int msg = sh.message[ai & 1], slices = msg & 15;
          last = msg & 256;
          const uint32_t up = abase + (ai & 1) * shp.abytes, h = up + (uint32_t)(shp.step_adapters * kProjTileN * a.rp);
          for (int i = 0; i < slices; ++i) {
            const uint32_t alo = core_lo(up + (uint32_t)(i * kProjTileN * a.rp));
            const uint32_t blo = ptx::umma_desc_lo(h + (uint32_t)(i * half * a.rp), (uint32_t)half * 16u);
            for (int k = 0; k < a.rp / 32; ++k) mma<kPair>(d, alo + k * 16, core_hi(8u * a.rp), blo + k * 2 * half, hhi, ida, 1u);
          }
          commit(&sh.aempty[ai & 1]);
        }
        if (ok) commit(&sh.tfull[ti & 1]);
      }
    }
  } else if (kFused && adapters && warp == 2 && blockIdx.x == 0) {
    look_over_requests(a);
  } else if (warp >= 4 && warp < 8 && adapters) {
    // The adapters of each unit's rows, then for each of its output tiles the operands of their steps.
    const int f = tid - 128;
    if (!kFused) ptx::grid_dependency_wait();
    auto rows_of = [&](int u, int ui) {                 // slot, live, list and n_list of unit u
      const int ub = ui & 1, row0 = u / shp.chunks * RT;
      if (!fill_all(wait(&sh.lfree[ub], ((ui >> 1) & 1) ^ 1))) return false;
      const bool scan = kFused && a.n_seg <= kScanRequests;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = f + i * kFill, row = row0 + r;
        if (r < RT) sh.slot[ub][r] = scan || row >= a.rows ? -2 : kFused ? slot_of_row(a, row) : slot_only(a.row_slot[row]);
      }
      fill_all(true);
      if (scan) {                                       // a warp reads 32 requests and writes the rows of those in the tile
        for (int q0 = f & ~31; q0 < a.n_seg; q0 += kFill) {
          const int q = q0 + lane;
          int lo = 0, hi = 0, s = -1;
          if (q < a.n_seg) {
            const int s0 = a.seg_start[q], s1 = a.seg_start[q + 1], ad = a.seg_adapter[q];
            lo = max(s0, row0);
            hi = min(min(s1, row0 + RT), a.rows);
            if (ad >= 0 && ad < a.max_adapters) s = ad;
          }
          for (uint32_t in = __ballot_sync(0xFFFFFFFFu, lo < hi); in; in &= in - 1) {
            const int from = __ffs((int)in) - 1;
            const int rlo = __shfl_sync(0xFFFFFFFFu, lo, from), rhi = __shfl_sync(0xFFFFFFFFu, hi, from), rs = __shfl_sync(0xFFFFFFFFu, s, from);
            for (int r = rlo + lane; r < rhi; r += 32) sh.slot[ub][r - row0] = rs;
          }
        }
        fill_all(true);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = f + i * kFill, s = r < RT ? sh.slot[ub][r] : -2;
        const uint32_t live = __ballot_sync(0xFFFFFFFFu, s != -2);
        if (lane == 0 && r < RT) sh.live[ub][r >> 5] = live;
        const uint32_t starts = __ballot_sync(0xFFFFFFFFu, r == 0 || (r < RT && sh.slot[ub][r - 1] != s));
        if (lane == 0 && r < RT) sh.starts[r >> 5] = starts;
      }
      fill_all(true);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = f + i * kFill;
        const uint32_t firsts = __ballot_sync(0xFFFFFFFFu, r < RT && first_of_slot(sh.slot[ub], sh.starts, r));
        if (lane == 0 && r < RT) sh.firsts[r >> 5] = firsts;
      }
      fill_all(true);
      // the list in the order of the rows: both CTAs of a pair walk it alike
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = f + i * kFill;
        int at = 0;
        for (int w = 0; w < (r >> 5) && w < RT / 32; ++w) at += __popc(sh.firsts[w]);
        if (r < RT) {
          const uint32_t word = sh.firsts[r >> 5];
          if (word >> lane & 1) sh.list[ub][at + __popc(word & ((1u << lane) - 1))] = sh.slot[ub][r];
          if (r == RT - 1) sh.n_list[ub] = at + __popc(word);
        }
      }
      fill_all(true);
      ptx::mbar_arrive(ptx::smem_u32(&sh.lready[ub]));
      return true;
    };
    int ai = 0, ui = 0, hi = 0;
    bool ok = unit0 >= shp.units || rows_of(unit0, 0);
    for (int u = unit0; ok && u < shp.units; u += unit_step, ++ui) {
      const int row0 = u / shp.chunks * RT, t0 = first_tile(u), t1 = last_tile(u), ub = ui & 1;
      const int n_list = sh.n_list[ub];
      int slot[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) slot[i] = f + i * kFill < half ? sh.slot[ub][part * half + f + i * kFill] : -2;
      if (u + unit_step < shp.units && !(ok = rows_of(u + unit_step, ui + 1))) break;   // a unit ahead
      if (kFused && n_list && !(ok = fill_all(wait(&sh.hready, hi++ & 1)))) break;
      for (int tn = t0; ok && tn < t1; ++tn) {
        int at = 0;
        do {
          const int ab = ai & 1, slices = min(shp.step_adapters, n_list - at);
          if (!(ok = fill_all(wait(&sh.aempty[ab], ((ai >> 1) & 1) ^ 1)))) break;
          ++ai;
          const uint32_t bar = ptx::smem_u32(&sh.afull[ab]), up = abase + ab * shp.abytes;
          uint8_t* const h = smem + (up - base) + shp.step_adapters * kProjTileN * a.rp;
          if (f == 0) {
            sh.message[ab] = slices | (at + slices >= n_list ? 256 : 0);
            if (slices) {
              const uint32_t bytes = (uint32_t)(kProjTileN * a.rp);
              ptx::mbar_expect_tx(bar, slices * bytes);
              for (int i = 0; i < slices; ++i)
                ptx::bulk_g2s(up + i * bytes, a.up + ((size_t)sh.list[ub][at + i] * a.tiles_n + stored_tile(tn)) * bytes, bytes, bar);
            } else {
              ptx::mbar_arrive(bar);
            }
          }
          for (int i = 0; i < slices; ++i) {
            const int s = sh.list[ub][at + i];
            for (int c = 0; c < a.rp / 16; c += 2) {    // 32 rank channels of two rows: loads first, then stores
              int4 t[2][2];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const bool mine = slot[e >> 1] == s;
                t[e >> 1][e & 1] = make_int4(0, 0, 0, 0);
                if (mine) t[e >> 1][e & 1] = __ldcg(reinterpret_cast<const int4*>(a.h + (size_t)(row0 + part * half + f + (e >> 1) * kFill) * a.rp) + c + (e & 1));
              }
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (f + (e >> 1) * kFill < half)
                  *reinterpret_cast<int4*>(h + ((i * (a.rp / 16) + c + (e & 1)) * half + f + (e >> 1) * kFill) * 16) = t[e >> 1][e & 1];
            }
          }
          ptx::fence_async_smem();
          ptx::mbar_arrive(bar);
          at += slices;
        } while (at < n_list);
      }
    }
    for (int i = 0; ok && i < 2; ++i, ++ai) ok = wait(&sh.aempty[ai & 1], ((ai >> 1) & 1) ^ 1);     // as given_back
  } else if (warp >= 8) {
    // A thread owns an output channel and walks over the rows. The exact requantisation runs on the half-rate integer
    // pipes (17 to 20 outputs per clock and SM with 16 warps, see the requantisation microbenchmark), so what is added to
    // it is kept small: the clip of an 8-bit type is the saturating pack, rows leave as words of four channels.
    const int q = warp & 3, cols = RT / (kEpiWarps / 4), c0 = ((warp - 8) >> 2) * cols;
    uint32_t* const stage = sh.out[warp - 8];
    int ti = 0, ui = 0;
    bool ok = true;
    auto sums = [&]() {
      ok = __all_sync(0xFFFFFFFFu, wait(&sh.tfull[ti & 1], (ti >> 1) & 1));
      ptx::tc_fence_after();
      return tmem + ((uint32_t)(q * 32) << 16) + (ti & 1) * RT + c0;
    };
    auto done = [&](uint64_t* bar) {
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (kPair) ptx::mbar_arrive_cluster(ptx::cluster_addr(ptx::smem_u32(bar), 0u));
        else ptx::mbar_arrive(ptx::smem_u32(bar));
      }
    };
    int4 rq_next = a.rq[stored_tile(first_tile(unit0)) * kProjTileN + q * 32 + lane];
    for (int u = unit0; ok && u < shp.units; u += unit_step, ++ui) {
      const int row0 = u / shp.chunks * RT, t0 = first_tile(u), t1 = last_tile(u), ub = ui & 1;
      if (adapters && !(ok = __all_sync(0xFFFFFFFFu, wait(&sh.lready[ub], (ui >> 1) & 1)))) break;
      if (kFused && adapters) {
        // The product's lanes are rank channels: those of one adapter would be work for a quarter of the warps (tensor
        // memory shows a warp 32 lanes), so copies of them stand in the other lanes, a share of the rows each.
        const int n_list = sh.n_list[ub], m = q * 32 + lane, j = m % a.rp;
        for (int g = 0; ok && g < n_list; g += per, ++ti) {
          const int n = min(per, n_list - g), copies = per / n, i = m / a.rp % n, copy = m / a.rp / n;
          const int slot = sh.list[ub][g + i];
          const int2 rq = a.down_rq[slot * a.rp + j];
          const uint32_t d = sums();
          if (!ok) break;
          for (int c = copy < copies ? copy * 16 : cols; c < cols; c += copies * 16) {
            uint32_t v[16];
            ptx::tmem_ld16(d + c, v);
            ptx::tmem_ld_wait16(v);
            store_rank(a.h + (size_t)(row0 + c0 + c) * a.rp + j, a.rp, v, rq, slot, sh.slot[ub] + c0 + c);
          }
          done(&sh.tempty[ti & 1]);
        }
        if (!ok) break;
        if (n_list) {                                   // each warp's h is written: to the warps that lay it out
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.hready));
        }
      }
      for (int tn = t0; ok && tn < t1; ++tn, ++ti) {
        const int n0 = tn * kProjTileN + q * 32, n = n0 + lane;
        const int4 rq = rq_next;
        {                                               // the next tile's constants
          const int un = u + unit_step;
          const int next = tn + 1 < t1 ? tn + 1 : un < shp.units ? first_tile(un) : tn;
          rq_next = a.rq[stored_tile(next) * kProjTileN + q * 32 + lane];
        }
        const long long add = (long long)(((unsigned long long)(uint32_t)rq.w << 32) | (uint32_t)rq.z);
        const int shift = max(rq.y - 1, 0);
        const bool words = sizeof(YT) == 1 && shp.vector_y && n0 + 32 <= a.n;
        const int first = words ? lane >> 3 << 2 : 0;  // rows first .. first + 3 of each 16 are this lane's, channels n0 + 4 (lane & 7) ..
        YT* y = (YT*)a.y + (long long)(row0 + c0 + first) * a.ldy + (words ? n0 + (lane & 7) * 4 : n);
        const uint32_t d = sums();
        if (!ok) break;
        for (int c = 0; c < cols; c += 32, y += 32 * a.ldy) {
          uint32_t v[2][16];
          ptx::tmem_ld16(d + c, v[0]);
          ptx::tmem_ld16(d + c + 16, v[1]);
          const int r = c0 + c, rest = a.rows - row0 - r;
          uint32_t rows32 = rest >= 32 ? 0xFFFFFFFFu : rest > 0 ? (1u << rest) - 1 : 0;    // the rows that are written, a bit each
          if (adapters) rows32 &= sh.live[ub][r >> 5];
          ptx::tmem_ld_wait16(v[0]);
          ptx::tmem_ld_wait16_nosync(v[1]);
          int o[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = requantised<kAnyShift>((int)v[e >> 4][e & 15], rq, add, shift);
          if (shp.clip) {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = min(max(o[e], a.lo), a.hi);
          }
          if (words) {                                  // four rows to a word, 32 x 32 of them transposed through shared memory
#pragma unroll
            for (int i = 0; i < 8; ++i) stage[i * 32 + lane] = pack4<YT>(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            __syncwarp();
            const int4 t0 = *reinterpret_cast<const int4*>(stage + lane * 4), t1 = *reinterpret_cast<const int4*>(stage + 128 + lane * 4);
            __syncwarp();
            uint32_t w[8];
            transpose4(t0, w);
            transpose4(t1, w + 4);
            YT* p = y;
            if (rows32 == 0xFFFFFFFFu) {
#pragma unroll
              for (int i = 0; i < 4; ++i, p += a.ldy) {
                *reinterpret_cast<uint32_t*>(p) = w[i];
                *reinterpret_cast<uint32_t*>(p + 16 * a.ldy) = w[4 + i];
              }
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i, p += a.ldy) {
                if (rows32 >> (first + i) & 1) *reinterpret_cast<uint32_t*>(p) = w[i];
                if (rows32 >> (16 + first + i) & 1) *reinterpret_cast<uint32_t*>(p + 16 * a.ldy) = w[4 + i];
              }
              __syncwarp();                             // these stores may have parted the lanes; the loads of the next step are the whole warp's
            }
          } else {
            if (n < a.n) {
              YT* p = y;
              if (sizeof(YT) == 1) {
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = min(max(o[e], YT(-1) < YT(0) ? -128 : 0), YT(-1) < YT(0) ? 127 : 255);
              }
              if (rows32 == 0xFFFFFFFFu) {
#pragma unroll
                for (int e = 0; e < 32; ++e, p += a.ldy) *p = (YT)o[e];
              } else {
#pragma unroll
                for (int e = 0; e < 32; ++e, p += a.ldy)
                  if (rows32 >> e & 1) *p = (YT)o[e];
              }
            }
            __syncwarp();
          }
        }
        done(&sh.tempty[ti & 1]);
      }
      if (ok && lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.lfree[ub]));
    }
  }
  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  if (kPair) {                                          // nothing of the pair reads or arrives in the other CTA any more
    ptx::cluster_arrive();
    ptx::cluster_wait();
  }
  if (warp == 2) {
    if (kPair) ptx::tmem_dealloc_pair(tmem, (uint32_t)shp.tmem_cols);
    else ptx::tmem_dealloc(tmem, (uint32_t)shp.tmem_cols);
  }
}

// ---- the projection of few rows ------------------------------------------------------------------------------------
// Where a tile per SM is not reached, the CTAs of a cluster share a tile: each multiplies a part of K, sends its int32
// sums to the CTA that owns the row (shared memory of the cluster) and finishes RT / S rows itself. There are few
// rows, mostly of different requests, so the adapters' products are dot products of 16 bytes here: an adapter
// step of the main kernel costs a tile's time whatever the number of rows that use it. Latency bounds it. One row, 1024 -> 4096, rank
// 16: 6.0 us with h (0.7 TB/s of weights); 48 rows, 2048 -> 2048, an adapter each: 9.7 us.
constexpr int kSplitThreads = 256;       // warp 0 copies, 1 MMAs, 2 tensor memory, 4-7 send the sums; all finish rows
constexpr int kSplitRing = 8;
constexpr int kSplitRows = 128;          // rows of a tile at most

struct SplitShared {
  uint64_t full[kSplitRing], empty[kSplitRing], tfull;
  uint32_t abort_flag, tmem;
};

struct SplitShape {
  int tile, ring, parts;                 // rows of a tile, stages of the ring, CTAs of a cluster (powers of two: tile, parts)
  int vector_y;                          // four neighbouring outputs lie on a 4 or 16-byte boundary
};

template <class YT, bool kAnyShift>
__global__ void __launch_bounds__(kSplitThreads, 1) proj_split_kernel(const __grid_constant__ CUtensorMap xmap, const ProjArgs a, const SplitShape shp) {
  extern __shared__ uint8_t raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  __shared__ SplitShared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int RT = shp.tile, ring = shp.ring, own = RT / shp.parts;       // rows that this CTA finishes
  const int part = (int)ptx::cluster_rank(), t = blockIdx.x / shp.parts;
  const int tn = t % a.tiles_n, row0 = t / a.tiles_n * RT;
  const int k0 = part * a.stages / shp.parts, k1 = (part + 1) * a.stages / shp.parts;
  const uint32_t stage_bytes = (uint32_t)(RT * kProjStage + kBytesW);
  if (tid == 0) {
    for (int i = 0; i < ring; ++i) {
      ptx::mbar_init(ptx::smem_u32(&sh.full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh.empty[i]), 1);
    }
    ptx::mbar_init(ptx::smem_u32(&sh.tfull), 1);
    ptx::mbar_init_fence();
    sh.abort_flag = 0;
  }
  // First phase of the cluster's barrier: every CTA runs before any of them writes into another. Tensor memory is given
  // back before the second: a CTA that kept it while another CTA of its cluster waits for tensor memory on its own SM
  // could lock up with another kernel's cluster.
  ptx::cluster_arrive();
  const uint32_t tmem_cols = (uint32_t)max(32, RT);
  if (warp == 2) ptx::tmem_alloc(ptx::smem_u32(&sh.tmem), tmem_cols);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t base = ptx::smem_u32(smem), tmem = sh.tmem;
  const int* const sums = reinterpret_cast<const int*>(smem + ring * stage_bytes);   // [parts][own][128]
  volatile uint32_t* abort_flag = &sh.abort_flag;

  if (warp == 0 && ptx::elect_one()) {
    const uint8_t* w = a.w + (size_t)tn * a.stages * kBytesW;
    Turn turn;
    for (int ks = k0; ks < k1; ++ks, turn.next(ring)) {
      const int s = turn.slot;
      if (!ptx::quick_wait(abort_flag, a.status, &sh.empty[s], turn.phase ^ 1, kSpinLimit)) break;
      const uint32_t st = base + s * stage_bytes, bar = ptx::smem_u32(&sh.full[s]);
      ptx::mbar_expect_tx(bar, stage_bytes);
      ptx::bulk_g2s(st + RT * kProjStage, w + (size_t)ks * kBytesW, kBytesW, bar);
      ptx::tile_g2s(st, &xmap, ks * kProjStage, row0, bar);
    }
    given_back(abort_flag, a.status, sh.empty, turn, ring);
  } else if (warp == 1 && ptx::elect_one()) {
    const uint32_t id = idesc((uint32_t)RT, a.x_unsigned);
    Turn turn;
    for (int ks = k0; ks < k1; ++ks, turn.next(ring)) {
      const int s = turn.slot;
      if (!ptx::quick_wait(abort_flag, a.status, &sh.full[s], turn.phase, kSpinLimit)) break;
      ptx::tc_fence_after();
      const uint32_t st = base + s * stage_bytes;
      stage_mmas(tmem, core_lo(st + RT * kProjStage), ptx::umma_desc_lo(st, 16u), id, min(4, (a.k - ks * kProjStage + 31) >> 5), ks == k0);
      ptx::umma_commit(ptx::smem_u32(&sh.empty[s]));
    }
    ptx::umma_commit(ptx::smem_u32(&sh.tfull));
  } else if (warp >= 4) {
    const int q = warp & 3;
    ptx::cluster_wait();
    const uint32_t dst = ptx::smem_u32(sums) + (uint32_t)(part * own * kProjTileN + q * 32 + lane) * 4u;
    if (__all_sync(0xFFFFFFFFu, ptx::quick_wait(abort_flag, a.status, &sh.tfull, 0u, kSpinLimit))) {
      ptx::tc_fence_after();
      for (int c = 0; c < RT; c += 16) {
        uint32_t v[16];
        ptx::tmem_ld16(tmem + ((uint32_t)(q * 32) << 16) + c, v);
        ptx::tmem_ld_wait16(v);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = c + e;
          ptx::st_cluster(ptx::cluster_addr(dst + (uint32_t)((r & (own - 1)) * kProjTileN * 4), (uint32_t)(r / own)), v[e]);
        }
      }
      ptx::tc_fence_before();
    }
  }
  if (warp < 4) ptx::cluster_wait();
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 2) ptx::tmem_dealloc(tmem, tmem_cols);
  ptx::cluster_arrive();
  const int n = tn * kProjTileN + lane * 4;                   // from here on a thread owns four neighbouring channels
  int4 rq[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) rq[i] = a.rq[n + i];
  if (a.n_seg) ptx::grid_dependency_wait();
  ptx::cluster_wait();
  for (int r = warp; r < own; r += kSplitThreads / 32) {
    const int row = row0 + part * own + r;
    if (row >= a.rows) break;
    const int slot_rank = a.n_seg ? a.row_slot[row] : -1;
    if (slot_rank == -2) continue;
    int4 v = make_int4(0, 0, 0, 0);
    for (int p = 0; p < shp.parts; ++p) {
      const int4 u = *reinterpret_cast<const int4*>(sums + (p * own + r) * kProjTileN + lane * 4);
      v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    int acc[4] = {v.x, v.y, v.z, v.w};
    if (slot_rank >= 0) {
      const int slot = slot_rank & ((1 << kSlotBits) - 1), chunks = ((slot_rank >> kSlotBits) + 15) >> 4;
      const int4* h = reinterpret_cast<const int4*>(a.h + (size_t)row * a.rp);
      const uint8_t* up = a.up + ((size_t)slot * a.tiles_n + tn) * kProjTileN * a.rp + (lane >> 1) * a.rp * 8 + (lane & 1) * 64;
      for (int c = 0; c < chunks; ++c) {
        const int4 hv = h[c];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = dot16<false>(*reinterpret_cast<const int4*>(up + c * 128 + i * 16), hv, acc[i]);
      }
    }
    int o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long add = (long long)(((unsigned long long)(uint32_t)rq[i].w << 32) | (uint32_t)rq[i].z);
      o[i] = min(max(requantised<kAnyShift>(acc[i], rq[i], add, max(rq[i].y - 1, 0)), a.lo), a.hi);
    }
    YT* y = (YT*)a.y + (long long)row * a.ldy + n;
    if (shp.vector_y && n + 4 <= a.n) {
      if (sizeof(YT) == 1)
        *reinterpret_cast<uint32_t*>(y) = pack4<YT>(o[0], o[1], o[2], o[3]);
      else
        *reinterpret_cast<int4*>(y) = make_int4(o[0], o[1], o[2], o[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < a.n) y[i] = (YT)o[i];
    }
  }
}

constexpr int kMaxSmem = 204 * 1024;      // beside 1 KB of alignment and the static part

int tiles_of(const ProjArgs& a, int tile) { return a.tiles_n * ((a.rows + tile - 1) / tile); }

// CTAs of a cluster of the kernel for few rows: as many as let all clusters run at once (one of 8 too many: 16 x 8192 -> 2048, 16
// tiles, takes 10.1 us with 8 and 6.7 with 4; 64 x 4096 -> 2048 with 64 requests 16.6 and 12.1), each with a stage of K.
int split_parts(const ProjArgs& a, int tile) {
  const int tiles = tiles_of(a, tile);
  int i = 0;
  while (i < 3 && tiles <= a.clusters[i + 1] && 2 << i <= a.stages) ++i;
  return 1 << i;
}

bool main_rings(const ProjArgs& a, int tile, bool fused, MainShape* s);
bool fuse_down(const ProjArgs& a);

// Different adapters that `rows` neighbouring rows use, as far as the host can tell: requests of even length.
long long adapters_of(const ProjArgs& a, int rows) {
  const long long most = std::min<long long>(a.n_seg, a.max_adapters);
  return std::max(1ll, std::min<long long>(most, ((long long)a.n_seg * std::min(rows, a.rows) + a.rows - 1) / a.rows));
}

// What down_rows_kernel takes beyond a launch, in ns: blocks of a row and eight rank channels.
long long down_rows_ns(const ProjArgs& a) { return (long long)a.rows * ((a.max_rank + 7) / 8) * (350 + 68 * a.k / 100) / 1000; }

// What down_tile_kernel takes beyond that: its latency and, much more, each further group of 128 / rp adapters of a tile. us of a
// call with h by rows and in tiles, 2048 -> 4096: 512 rows, rank 16, 4 requests 14.9 and 18.2; 1024 rows, 32, 8 requests 20.6 and
// 18.6; 1024 rows, 128, 8 requests 43.3 and 20.2; 1024 rows, 32, 128 requests 30.8 and 49.5; 2048 rows, 16, 512 requests 53.1 and 66.6.
long long down_tiles_ns(const ProjArgs& a) {
  const long long per = kProjTileN / a.rp, groups = (adapters_of(a, kDownRows) + per - 1) / per;
  const long long waves = ((a.rows + kDownRows - 1) / kDownRows + 3 * a.sms - 1) / (3 * a.sms);
  return waves * (2500 + (groups - 1) * (1500 + 3 * a.k));
}

// Rows of a tile of the kernel for few rows, 0 where it is the slower one. Both times are modelled in ns, from measurements
// at K 256, 1024 and 4096, rank 0, 16 and 64, 0 to 512 requests. The few rows' kernel: a tile's rows are sent, a CTA's own rows are
// finished one after another. The persistent one: K, which it does not split, and an adapter step for each adapter of a tile. us, few
// rows' kernel and persistent, for 16, 64, 128, 256, 512 rows: 1024 -> 4096 without adapters 4.8 and 6.5, 6.0 and 6.5, 8.2
// and 6.5, 9.0 and 6.6, 11.7 and 7.0; with 8 requests of rank 16: 7.1 and 22.6, 9.6 and 22.5, 12.2 and 22.3, 16.2 and 15.5, 24.0
// and 13.6; 4096 -> 4096 with 8: 9.8 and 18.5, 12.1 and 21.1, 15.4 and 21.7, 20.5 and 22.2, 31.4 and 21.2.
int split_tile(const ProjArgs& a) {
  int t = 16;
  while (t < kSplitRows && t < a.rows) t *= 2;
  if (tiles_of(a, t) > a.sms) return 0;
  const int parts = split_parts(a, t), own = t / parts;
  const bool fused = fuse_down(a);
  long long split = 3600 + 25 * (t + own) + 16 * a.k / (10 * parts), main = fused ? 4500 + 2 * a.k : 6500 + 22 * a.k / 10;
  if (a.n_seg) {
    split += 1400 + 6 * std::min(a.k, 1024) / 10 + own * (30 + 5 * a.max_rank / 2) + down_rows_ns(a);
    main += fused ? 4600 + 19 * a.k / 10 : 2600 + 30 * a.rp + std::min(down_rows_ns(a), down_tiles_ns(a));
    main += (fused ? 30 : 16) * a.rp * (adapters_of(a, kSplitRows) - 1);
  }
  return split <= main ? t : 0;
}

// Shared memory of the persistent kernel with tiles of `tile` rows: false if it does not fit.
bool main_rings(const ProjArgs& a, int tile, bool fused, MainShape* s) {
  const int half = fused ? tile : tile / 2, x = half * kProjStage;
  for (s->step_adapters = a.rp == 32 ? 2 : 1; s->step_adapters >= 1; --s->step_adapters) {
    s->abytes = (kProjTileN + half) * a.rp * s->step_adapters;
    const int room = kMaxSmem - (a.n_seg ? 2 * s->abytes : 0);
    if (fused) {
      for (int sets = 2; sets >= 1; --sets) {
        s->xring = sets * a.stages;
        s->wring = std::min(kMaxRing, (room - s->xring * x) / kBytesW);
        if (s->xring <= kMaxX && s->wring >= 3) return true;
      }
    } else {
      s->xring = s->wring = std::min(kMaxRing, room / (x + kBytesW));
      if (s->xring >= 2) return true;
    }
  }
  return false;
}

// h within the projection's own kernel, or before it.
bool fuse_down(const ProjArgs& a) {
  MainShape s;
  return main_rings(a, kMaxTile / 2, true, &s);
}

// Rows of a tile and output tiles of a unit of the persistent kernel: what costs the least. The cost is the units per SM
// (one at least) times a unit's items (its output tiles, and one more for h with adapters) times an item's cost, its rows
// and as much as 128 rows more. Measured, us for (rows, chunk) = (128, 1) (128, 2) (128, 4) (256, 1) (256, 2) (256, 4):
// 65536 x 512 -> 512: 76 53 46 49 40 35; 32768 x 256 -> 256: 25 18 18 18 14 14; 20011 x 173 -> 109 (one output tile): 18.6 and 21.6.
void main_tiles(const ProjArgs& a, int* tile, int* chunk) {
  const bool fused = fuse_down(a);
  long long least = LLONG_MAX;
  if (!fused) {                                         // a pair's MMA has 256 rows at its best
    *tile = kMaxTile;
    *chunk = 1;
    return;
  }
  for (int t = kMaxTile; t >= kMaxTile / 2; t /= 2) {
    const long long row_tiles = (a.rows + t - 1) / t;
    MainShape s;
    if (!main_rings(a, t, fused, &s)) continue;
    for (int c = 1; c <= a.tiles_n; ++c) {
      const long long units = row_tiles * ((a.tiles_n + c - 1) / c);
      const long long cost = std::max<long long>(units, a.sms) * (c + (a.n_seg ? 1 : 0)) * (t + 128);
      if (cost < least) {
        least = cost;
        *tile = t;
        *chunk = c;
      }
    }
  }
}

int row_tile(const ProjArgs& a) {
  int tile = split_tile(a), chunk;
  if (!tile) main_tiles(a, &tile, &chunk);
  return tile;
}

template <class... Params, class... Given>
cudaError_t launch_tiles(void (*kernel)(Params...), int grid, int cluster, int threads, size_t smem, bool follows_down, cudaStream_t stream,
                         const Given&... given) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = follows_down ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, given...);
}

template <class YT, bool kAnyShift>
cudaError_t launch_main(const ProjArgs& a, const CUtensorMap& map, const CUtensorMap& w_map, cudaStream_t stream) {
  const int tile = row_tile(a), tiles = tiles_of(a, tile), stage = tile * kProjStage + kBytesW;
  const uintptr_t y = reinterpret_cast<uintptr_t>(a.y);
  if (split_tile(a)) {
    SplitShape s;
    s.tile = tile;
    s.parts = split_parts(a, tile);
    const int sums = tile * kProjTileN * 4, most = (a.stages + s.parts - 1) / s.parts;
    s.ring = std::min(std::min(kSplitRing, most), (kMaxSmem - sums) / stage);
    s.vector_y = a.ldy % 4 == 0 && y % (4 * a.y_bytes) == 0;
    return launch_tiles(proj_split_kernel<YT, kAnyShift>, tiles * s.parts, s.parts, kSplitThreads, (size_t)(s.ring * stage + sums + 1024),
                        a.n_seg != 0, stream, map, a, s);
  }
  MainShape s;
  s.tile = tile;
  s.tmem_cols = 2 * tile;
  s.vector_y = a.y_bytes == 1 && a.ldy % 4 == 0 && y % 4 == 0;
  const int lo = a.y_type == IODF_I8 ? -128 : a.y_type == IODF_U8 ? 0 : INT_MIN, hi = a.y_type == IODF_I8 ? 127 : a.y_type == IODF_U8 ? 255 : INT_MAX;
  s.clip = a.lo > lo || a.hi < hi;
  const bool fused = fuse_down(a);
  main_rings(a, tile, fused, &s);
  const int row_tiles = (a.rows + tile - 1) / tile;
  int unused;
  main_tiles(a, &unused, &s.chunk);
  const int ctas = fused ? 1 : 2;                       // of a unit
  s.chunks = (a.tiles_n + ctas * s.chunk - 1) / (ctas * s.chunk);
  s.units = row_tiles * s.chunks;
  return launch_tiles(fused ? proj_tile_kernel<YT, kAnyShift, true> : proj_tile_kernel<YT, kAnyShift, false>,
                      std::min(s.units, a.sms / ctas) * ctas, ctas, kMainThreads,
                      (size_t)(s.xring * tile / ctas * kProjStage + s.wring * kBytesW + (a.n_seg ? 2 * s.abytes : 0) + 1024),
                      a.n_seg != 0 && !fused, stream, map, w_map, a, s);
}

template <class YT, bool kAnyShift>
cudaError_t configure() {
  const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaFuncSetAttribute(proj_tile_kernel<YT, kAnyShift, false>, attr, kMaxSmem + 1024);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(proj_tile_kernel<YT, kAnyShift, true>, attr, kMaxSmem + 1024);
  return e == cudaSuccess ? cudaFuncSetAttribute(proj_split_kernel<YT, kAnyShift>, attr, kMaxSmem + 1024) : e;
}

}  // namespace

cudaError_t configure_proj_kernels(int device, ProjArgs* a) {
  cudaError_t e = cudaFuncSetAttribute(down_tile_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kDownRing * kDownStageBytes + 1024);
  if (e == cudaSuccess) e = configure<int8_t, false>();
  if (e == cudaSuccess) e = configure<int8_t, true>();
  if (e == cudaSuccess) e = configure<uint8_t, false>();
  if (e == cudaSuccess) e = configure<uint8_t, true>();
  if (e == cudaSuccess) e = configure<int, false>();
  if (e == cudaSuccess) e = configure<int, true>();
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&a->sms, cudaDevAttrMultiProcessorCount, device);
  for (int i = 0; i < 4 && e == cudaSuccess; ++i) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1u << i);
    cfg.blockDim = dim3(kSplitThreads);
    cfg.dynamicSmemBytes = kMaxSmem + 1024;             // one CTA per SM
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1u << i;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&a->clusters[i], proj_split_kernel<int8_t, false>, &cfg);
  }
  return e;
}

bool proj_down_tiles(const ProjArgs& a) {
  return a.n_seg && !split_tile(a) && !fuse_down(a) && down_tiles_ns(a) < down_rows_ns(a);
}

int proj_x_rows(const ProjArgs& a) { return split_tile(a) || fuse_down(a) ? row_tile(a) : row_tile(a) / 2; }

cudaError_t launch_proj(const ProjArgs& a, const void* x_map, const void* x_map_down, const void* w_map, cudaStream_t stream) {
  if (a.n_seg && (split_tile(a) || !fuse_down(a))) {
    if (!proj_down_tiles(a)) {
      const dim3 grid((unsigned)a.rows, (unsigned)(a.rp / 8));
      if (a.x_unsigned) down_rows_kernel<true><<<grid, 128, 0, stream>>>(a);
      else down_rows_kernel<false><<<grid, 128, 0, stream>>>(a);
    } else {
      const int tiles = (a.rows + kDownRows - 1) / kDownRows, ring = tiles > a.sms ? 2 : kDownRing;
      down_tile_kernel<<<tiles, kDownThreads, ring * kDownStageBytes + 1024, stream>>>(*static_cast<const CUtensorMap*>(x_map_down), a, ring);
    }
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  const CUtensorMap &map = *static_cast<const CUtensorMap*>(x_map), &wm = *static_cast<const CUtensorMap*>(w_map);
  if (a.y_type == IODF_I8) return a.any_shift ? launch_main<int8_t, true>(a, map, wm, stream) : launch_main<int8_t, false>(a, map, wm, stream);
  if (a.y_type == IODF_U8) return a.any_shift ? launch_main<uint8_t, true>(a, map, wm, stream) : launch_main<uint8_t, false>(a, map, wm, stream);
  return a.any_shift ? launch_main<int, true>(a, map, wm, stream) : launch_main<int, false>(a, map, wm, stream);
}

}  // namespace iodf
