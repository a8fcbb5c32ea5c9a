// C ABI of the single integer layers (include/iodf.h): the projection with low-rank adapters and the norms
// before and after a block. Host side only: checks, packing, device buffers, launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdlib>
#include <cstring>
#include <exception>
#include <new>
#include <vector>

#include "../../include/iodf.h"
#include "api_common.h"
#include "norm_kernel.h"
#include "proj_kernel.h"
#include "refine.h"

using namespace iodf;

struct iodf_proj {
  int device = 0;
  EncodeTiled encode = nullptr;
  CUtensorMap w_map;
  uint32_t max_rows = 0, max_adapters = 0, max_rank = 0;
  int amax = 128;                            // largest |x|
  ProjArgs args{};
  std::vector<int64_t> room;                 // per output channel: int32 range left beside the shared part
  void* d_mem = nullptr;                     // one allocation for everything below args
};

struct iodf_norm {
  int device = 0;
  NormArgs args{};
  int32_t* d_consts = nullptr;
};

namespace {

bool capturing(cudaStream_t s) {
  cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
  return cudaStreamIsCapturing(s, &st) != cudaSuccess || st != cudaStreamCaptureStatusNone;
}

// Sum of |w| of one row (at most 32768 * 128).
int magnitude(const int8_t* w, size_t n) {
  int sum = 0;
  for (size_t i = 0; i < n; ++i) sum += std::abs((int)w[i]);
  return sum;
}

// A row of K channels of an operand of `rows` rows, cut into stages.
void pack_row(uint8_t* dst, size_t rows, size_t row, const int8_t* src, size_t K) {
  for (size_t k = 0; k < K; k += 16)
    std::memcpy(dst + k / kProjStage * rows * kProjStage + core_offset(row, k % kProjStage, kProjStage), src + k, std::min<size_t>(16, K - k));
}

// uint8 [rows][cols], row stride `ld`, boxes of one stage x box_rows rows
bool tile_map(const iodf_proj& p, const void* base, uint64_t cols, uint64_t rows, uint64_t ld, uint32_t box_rows, bool swizzle, CUtensorMap* out) {
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {ld};
  const cuuint32_t box[2] = {(cuuint32_t)kProjStage, box_rows}, steps[2] = {1, 1};
  return p.encode(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr uint32_t kMaxChannels = 32768, kMaxRank = 128, kMaxSlots = 65536, kMaxNormChannels = 8192, kMaxPlanes = 256;

int create_proj(const iodf_proj_desc& d, const int8_t* weights, size_t wn, const int32_t* requant, size_t rn, int device,
                iodf_proj& p) {
  const iodf_layer_desc& L = d.layer;
  if (L.c_in < 1 || L.c_out < 1 || (L.k != 1 && L.k != 3)) return IODF_EINVAL;
  if (L.k != 1 || L.c_in > kMaxChannels || L.c_out > kMaxChannels) return IODF_EUNSUPPORTED;
  if (d.x_type != IODF_I8 && d.x_type != IODF_U8) return IODF_EINVAL;
  if (d.y_type != IODF_I8 && d.y_type != IODF_U8 && d.y_type != IODF_I32) return IODF_EINVAL;
  if (d.max_rows < 1 || d.max_rows > (1u << 30) || d.max_adapters > kMaxSlots || d.max_rank > kMaxRank) return IODF_EINVAL;
  if (d.max_adapters && d.max_rank < 1) return IODF_EINVAL;
  const size_t K = L.c_in, N = L.c_out;
  if (L.weight_off > wn || N * K > wn - L.weight_off) return IODF_EINVAL;
  if (L.requant_off > rn || 3 * N > rn - L.requant_off) return IODF_EINVAL;
  const int8_t* w = weights + L.weight_off;
  const int32_t *bias = requant + L.requant_off, *m0 = bias + N, *s = m0 + N;
  for (size_t n = 0; n < N; ++n)
    if (m0[n] < (1 << 30) || s[n] < 0 || s[n] > 31) return IODF_EINVAL;
  int lo = INT32_MIN, hi = INT32_MAX;
  if (L.has_clamp) {
    if (L.clamp_lo > L.clamp_hi) return IODF_EINVAL;
    lo = L.clamp_lo;
    hi = L.clamp_hi;
  }
  if (L.relu) lo = std::min(std::max(lo, 0), hi);
  if (d.y_type == IODF_I8 && (lo < -128 || hi > 127)) return IODF_EINVAL;
  if (d.y_type == IODF_U8 && (lo < 0 || hi > 255)) return IODF_EINVAL;
  p.amax = d.x_type == IODF_U8 ? 255 : 128;
  p.room.resize(N);
  for (size_t n = 0; n < N; ++n) {
    p.room[n] = 0x7FFFFFFFll - ((int64_t)magnitude(w + n * K, K) * p.amax + std::llabs((long long)bias[n]));
    if (p.room[n] < 0) return IODF_EOVERFLOW;
  }

  const size_t S = kProjStage, stages = (K + S - 1) / S, tiles = (N + kProjTileN - 1) / kProjTileN, slots = d.max_adapters;
  const size_t R = d.max_rank <= 32 ? 32 : d.max_rank <= 64 ? 64 : 128;
  std::vector<uint8_t> wp(tiles * stages * kProjTileN * S, 0);
  std::vector<int4> rq(tiles * kProjTileN, make_int4(1 << 30, 1, 0, 0));
  for (size_t n = 0; n < N; ++n) {
    pack_row(&wp[n / kProjTileN * stages * kProjTileN * S], kProjTileN, n % kProjTileN, w + n * K, K);
    p.args.any_shift |= s[n] == 0;
    const int64_t add = (int64_t)bias[n] * m0[n] + (1ll << (30 + s[n]));
    rq[n] = make_int4(m0[n], s[n], (int)(uint32_t)add, (int)(uint32_t)((uint64_t)add >> 32));
  }

  // one device allocation, cut up
  size_t total = 0;
  auto part = [&](size_t bytes) {
    const size_t at = total;
    total += up_to(std::max<size_t>(bytes, 1), 256);
    return at;
  };
  const size_t o_w = part(wp.size()), o_rq = part(16 * rq.size()), o_down = part(slots * R * stages * S), o_drq = part(8 * slots * R),
               o_up = part(slots * tiles * kProjTileN * R), o_rank = part(4 * slots), o_h = part(slots ? d.max_rows * R : 0),
               o_slot = part(4 * (size_t)d.max_rows), o_status = part(8);
  p.device = device;
  p.max_rows = d.max_rows;
  p.max_adapters = d.max_adapters;
  p.max_rank = d.max_rank;
  OnDevice on(device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  p.encode = tensor_map_encoder();
  if (!p.encode) return IODF_ECUDA;
  cudaError_t e = configure_proj_kernels(device, &p.args);
  if (e == cudaSuccess) e = cudaMalloc(&p.d_mem, total);
  if (e != cudaSuccess) return status_of(e);
  uint8_t* m = static_cast<uint8_t*>(p.d_mem);
  e = cudaMemcpy(m + o_w, wp.data(), wp.size(), cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaMemcpy(m + o_rq, rq.data(), 16 * rq.size(), cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaMemset(m + o_down, 0, o_h - o_down);     // an empty slot adds nothing: all zeros
  if (e == cudaSuccess) e = cudaMemset(m + o_status, 0, 8);
  // A copy from pageable memory is only known to have left it: the first call may be on a stream that does not wait for the rest.
  if (e == cudaSuccess) e = cudaStreamSynchronize(0);
  if (e != cudaSuccess) return status_of(e);
  ProjArgs& a = p.args;
  a.k = (int)K;
  a.n = (int)N;
  a.stages = (int)stages;
  a.tiles_n = (int)tiles;
  a.x_unsigned = d.x_type == IODF_U8;
  a.y_type = (int)d.y_type;
  a.y_bytes = d.y_type == IODF_I32 ? 4 : 1;
  a.lo = lo;
  a.hi = hi;
  a.max_adapters = (int)slots;
  a.max_rank = (int)d.max_rank;
  a.rp = (int)R;
  a.w = m + o_w;
  a.rq = reinterpret_cast<const int4*>(m + o_rq);
  a.down = m + o_down;
  a.down_rq = reinterpret_cast<const int2*>(m + o_drq);
  a.up = m + o_up;
  a.rank = reinterpret_cast<const int*>(m + o_rank);
  a.h = reinterpret_cast<int8_t*>(m + o_h);
  a.row_slot = reinterpret_cast<int*>(m + o_slot);
  a.status = reinterpret_cast<uint32_t*>(m + o_status);
  if (!tile_map(p, a.w, S, tiles * stages * kProjTileN, S, kProjTileN, false, &p.w_map)) return IODF_ECUDA;
  return IODF_OK;
}

int set_adapter(iodf_proj& p, uint32_t slot, uint32_t rank, const int8_t* down, const int32_t* rq, const int8_t* up,
                cudaStream_t stream) {
  const size_t K = p.args.k, N = p.args.n, R = p.args.rp, S = kProjStage;
  const size_t dbytes = R * p.args.stages * S, ubytes = (size_t)p.args.tiles_n * kProjTileN * R;
  for (uint32_t j = 0; j < rank; ++j) {
    if (rq[j] < (1 << 30) || rq[rank + j] < 0 || rq[rank + j] > 31) return IODF_EINVAL;
    if ((int64_t)magnitude(down + j * K, K) * p.amax > 0x7FFFFFFFll) return IODF_EOVERFLOW;
  }
  for (size_t n = 0; n < N; ++n) {
    if ((int64_t)magnitude(up + n * rank, rank) * 128 > p.room[n]) return IODF_EOVERFLOW;
  }
  std::vector<uint8_t> dp(dbytes, 0), upp(ubytes, 0);
  std::vector<int2> q(R, make_int2(1 << 30, 0));
  for (uint32_t j = 0; j < rank; ++j) {
    pack_row(dp.data(), R, j, down + j * K, K);
    q[j] = make_int2(rq[j], rq[rank + j]);
  }
  for (size_t n = 0; n < N; ++n)
    for (uint32_t j = 0; j < rank; ++j)
      upp[n / kProjTileN * kProjTileN * R + core_offset(n % kProjTileN, j, R)] = (uint8_t)up[n * rank + j];
  const int rk = (int)rank;
  OnDevice on(p.device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  if (capturing(stream)) return IODF_EINVAL;
  const ProjArgs& a = p.args;
  cudaError_t e = cudaMemcpyAsync(const_cast<uint8_t*>(a.down) + slot * dbytes, dp.data(), dbytes, cudaMemcpyHostToDevice, stream);
  if (e == cudaSuccess) e = cudaMemcpyAsync(const_cast<int2*>(a.down_rq) + slot * R, q.data(), 8 * R, cudaMemcpyHostToDevice, stream);
  if (e == cudaSuccess) e = cudaMemcpyAsync(const_cast<uint8_t*>(a.up) + slot * ubytes, upp.data(), ubytes, cudaMemcpyHostToDevice, stream);
  if (e == cudaSuccess) e = cudaMemcpyAsync(const_cast<int*>(a.rank) + slot, &rk, 4, cudaMemcpyHostToDevice, stream);
  const cudaError_t e2 = cudaStreamSynchronize(stream);      // the arrays above live until here
  return status_of(e != cudaSuccess ? e : e2);
}

// Rows of `bytes` bytes at a stride, two of them: do they share memory? Of rows that lie within each other at one stride (columns of a
// wider matrix) it is known; at two strides they count as sharing it.
bool rows_overlap(const void* p, size_t pbytes, size_t pstride, const void* q, size_t qbytes, size_t qstride, size_t rows) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  if (a + (rows - 1) * pstride + pbytes <= b || b + (rows - 1) * qstride + qbytes <= a) return false;
  if (pstride != qstride || rows == 1) return true;
  const size_t at = b >= a ? (b - a) % pstride : (pstride - (a - b) % pstride) % pstride;      // of q's rows in p's
  return at < pbytes || at + qbytes > pstride;
}

// a: the handle's arguments, with a workspace and status words that may be another's
int proj_forward(const iodf_proj& p, ProjArgs a, const void* x, size_t ldx, int rows, const int32_t* seg_start, const int32_t* seg_adapter,
                 int n_seg, void* y, size_t ldy, cudaStream_t stream) {
  if (rows < 0 || (uint32_t)rows > p.max_rows || n_seg < 0) return IODF_EINVAL;
  if (rows == 0) return IODF_OK;
  if (!x || !y || (n_seg && (!seg_start || !seg_adapter))) return IODF_EINVAL;
  if (!aligned(x, 16) || ldx % 16 || ldx < (size_t)a.k || ldx >= (1ull << 40)) return IODF_EINVAL;
  if (!aligned(y, (size_t)a.y_bytes) || ldy < (size_t)a.n || ldy >= (1ull << 40)) return IODF_EINVAL;
  if (!aligned(seg_start, 4) || !aligned(seg_adapter, 4)) return IODF_EINVAL;
  // tiles are written while others are still read
  if (rows_overlap(x, (size_t)a.k, ldx, y, (size_t)a.n * a.y_bytes, ldy * a.y_bytes, (size_t)rows)) return IODF_EINVAL;
  a.x = static_cast<const uint8_t*>(x);
  a.ldx = (long long)ldx;
  a.y = y;
  a.ldy = (long long)ldy;
  a.seg_start = seg_start;
  a.seg_adapter = seg_adapter;
  a.n_seg = n_seg;
  a.rows = rows;
  OnDevice on(p.device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  CUtensorMap map, map_down;
  if (!tile_map(p, x, (uint64_t)a.k, (uint64_t)rows, ldx, (uint32_t)proj_x_rows(a), true, &map) ||
      (proj_down_tiles(a) && !tile_map(p, x, (uint64_t)a.k, (uint64_t)rows, ldx, kProjDownRows, true, &map_down)))
    return IODF_ECUDA;
  return status_of(launch_proj(a, &map, &map_down, &p.w_map, stream));
}

bool norm_kind(uint32_t k) { return k == IODF_NORM_RMS || k == IODF_NORM_CENTRED; }

int create_norm(const iodf_norm_desc& d, int device, iodf_norm& nm) {
  const uint32_t C = d.channels;
  if (C < 1) return IODF_EINVAL;
  if (C > kMaxNormChannels) return IODF_EUNSUPPORTED;
  if (d.res_type != IODF_I16 && d.res_type != IODF_I32) return IODF_EINVAL;
  if (d.block_type && d.block_type != IODF_I8 && d.block_type != IODF_I32) return IODF_EINVAL;
  if ((d.post_norm && !norm_kind(d.post_norm)) || (d.pre_norm && !norm_kind(d.pre_norm))) return IODF_EINVAL;
  if (!d.block_type && (d.post_norm || !d.pre_norm)) return IODF_EINVAL;
  if ((d.post_norm || d.pre_norm) && (d.eps < 1 || d.eps > (1ull << 60))) return IODF_EINVAL;
  if (d.block_type) {
    const int lim = d.res_type == IODF_I16 ? 1 << 15 : 1 << 23;
    if (!d.mult || d.shift < 1 || d.shift > 31) return IODF_EINVAL;
    if (d.res_lo > d.res_hi || d.res_lo < -lim || d.res_hi > lim - 1) return IODF_EINVAL;
    for (uint32_t c = 0; c < C; ++c)
      if (d.mult[c] == INT32_MIN) return IODF_EINVAL;
  }
  if (d.pre_norm) {
    if (!d.n_mult || !d.n_bias || d.n_shift < 1 || d.n_shift > 31 || d.n_lo > d.n_hi) return IODF_EINVAL;
    if (d.n_type != IODF_I8 && d.n_type != IODF_U8) return IODF_EINVAL;
    if (d.n_type == IODF_I8 ? (d.n_lo < -128 || d.n_hi > 127) : (d.n_lo < 0 || d.n_hi > 255)) return IODF_EINVAL;
    for (uint32_t c = 0; c < C; ++c)
      if (d.n_mult[c] == INT32_MIN || d.n_bias[c] <= -(1 << 30) || d.n_bias[c] >= (1 << 30)) return IODF_EINVAL;
  }
  const size_t cp = up_to(C, 64);               // tables end on a whole vector
  std::vector<int32_t> tab(3 * cp, 0);
  if (d.block_type) std::copy(d.mult, d.mult + C, tab.begin());
  if (d.pre_norm) {
    std::copy(d.n_mult, d.n_mult + C, tab.begin() + cp);
    std::copy(d.n_bias, d.n_bias + C, tab.begin() + 2 * cp);
  }
  nm.device = device;
  OnDevice on(device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  cudaError_t e = cudaMalloc(&nm.d_consts, 4 * tab.size());
  if (e == cudaSuccess) e = cudaMemcpy(nm.d_consts, tab.data(), 4 * tab.size(), cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaStreamSynchronize(0);        // the copy may still be on its way, as in create_proj
  if (e != cudaSuccess) return status_of(e);
  NormArgs& a = nm.args;
  a.channels = (int)C;
  a.res_i16 = d.res_type == IODF_I16;
  a.has_block = d.block_type != 0;
  a.block_i8 = d.block_type == IODF_I8;
  a.post = (int)d.post_norm;
  a.pre = (int)d.pre_norm;
  a.shift = d.shift;
  a.n_shift = d.n_shift;
  a.res_lo = d.res_lo;
  a.res_hi = d.res_hi;
  a.n_lo = d.n_lo;
  a.n_hi = d.n_hi;
  a.n_type = (int)d.n_type;
  a.n_full = d.n_type == IODF_I8 ? d.n_lo == -128 && d.n_hi == 127 : d.n_lo == 0 && d.n_hi == 255;
  a.eps = d.eps;
  a.mult = nm.d_consts;
  a.n_mult = nm.d_consts + cp;
  a.n_bias = nm.d_consts + 2 * cp;
  return IODF_OK;
}

bool good_view(const iodf_view& v, uint32_t channels) {
  const uint64_t big = 1ull << 40;
  if (v.pixels < 1 || v.pixels > big || v.image_stride > big || v.channel_stride > big || v.pixel_stride > big) return false;
  return v.channel_stride == 1 || (v.pixel_stride == 1 && channels <= kMaxPlanes);
}

// True if no two of rows x channels elements share a place, as far as the strides show it: in ascending order each is at
// least the extent of what it steps over.
bool apart(const iodf_view& v, uint64_t rows, uint64_t channels) {
  struct Dim { uint64_t n, stride; } d[3] = {{channels, v.channel_stride}, {std::min<uint64_t>(v.pixels, rows), v.pixel_stride},
                                             {(rows + v.pixels - 1) / v.pixels, v.image_stride}};
  std::sort(d, d + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  uint64_t extent = 1;
  for (const Dim& e : d) {
    if (e.n == 1) continue;
    if (e.stride < extent) return false;
    extent += e.stride * (e.n - 1);
  }
  return true;
}

ViewArgs view_args(const iodf_view& v) {
  return {(long long)v.pixels, (long long)v.image_stride, (long long)v.channel_stride, (long long)v.pixel_stride};
}

}  // namespace

extern "C" {

int iodf_proj_create(const iodf_proj_desc* desc, const int8_t* weights, size_t weights_count, const int32_t* requant,
                     size_t requant_count, int device, iodf_proj** out) {
  if (!desc || !weights || !requant || !out) return IODF_EINVAL;
  *out = nullptr;
  if (desc->abi_version != IODF_ABI_VERSION) return IODF_EVERSION;
  iodf_proj* p = new (std::nothrow) iodf_proj();
  if (!p) return IODF_ENOMEM;
  int rc;
  try {
    rc = create_proj(*desc, weights, weights_count, requant, requant_count, device, *p);
  } catch (const std::exception&) {              // out of host memory, or a size beyond what a vector may have
    rc = IODF_ENOMEM;
  }
  if (rc != IODF_OK) {
    iodf_proj_destroy(p);
    return rc;
  }
  *out = p;
  return IODF_OK;
}

void iodf_proj_destroy(iodf_proj* p) {
  if (!p) return;
  if (p->d_mem) {
    OnDevice on(p->device);
    cudaFree(p->d_mem);
  }
  delete p;
}

int iodf_proj_set_adapter(iodf_proj* p, uint32_t slot, uint32_t rank, const int8_t* down, const int32_t* down_requant,
                          const int8_t* up, void* cuda_stream) {
  if (!p || slot >= p->max_adapters || rank > p->max_rank) return IODF_EINVAL;
  if (rank && (!down || !down_requant || !up)) return IODF_EINVAL;
  try {
    return set_adapter(*p, slot, rank, down, down_requant, up, (cudaStream_t)cuda_stream);
  } catch (const std::exception&) {
    return IODF_ENOMEM;
  }
}

int iodf_proj_forward(iodf_proj* p, const void* x, size_t ldx, int rows, const int32_t* seg_start,
                      const int32_t* seg_adapter, int n_seg, void* y, size_t ldy, void* cuda_stream) {
  return p ? proj_forward(*p, p->args, x, ldx, rows, seg_start, seg_adapter, n_seg, y, ldy, (cudaStream_t)cuda_stream) : IODF_EINVAL;
}

int iodf_proj_check(iodf_proj* p, void* cuda_stream, uint32_t* bad_requests) {
  if (!p) return IODF_EINVAL;
  if (bad_requests) *bad_requests = 0;
  OnDevice on(p->device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  uint32_t st[2] = {0, 0};
  cudaError_t e = cudaStreamSynchronize((cudaStream_t)cuda_stream);
  if (e == cudaSuccess) e = cudaMemcpy(st, p->args.status, 8, cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && (st[0] || st[1])) e = cudaMemset(p->args.status, 0, 8);
  if (e == cudaSuccess) e = cudaStreamSynchronize(0);
  if (e != cudaSuccess) return IODF_ECUDA;
  if (bad_requests) *bad_requests = st[1];
  return st[0] ? IODF_ETIMEOUT : st[1] ? IODF_EDATA : IODF_OK;
}

int iodf_norm_create(const iodf_norm_desc* desc, int device, iodf_norm** out) {
  if (!desc || !out) return IODF_EINVAL;
  *out = nullptr;
  if (desc->abi_version != IODF_ABI_VERSION) return IODF_EVERSION;
  iodf_norm* nm = new (std::nothrow) iodf_norm();
  if (!nm) return IODF_ENOMEM;
  int rc;
  try {
    rc = create_norm(*desc, device, *nm);
  } catch (const std::exception&) {              // out of host memory, or a size beyond what a vector may have
    rc = IODF_ENOMEM;
  }
  if (rc != IODF_OK) {
    iodf_norm_destroy(nm);
    return rc;
  }
  *out = nm;
  return IODF_OK;
}

void iodf_norm_destroy(iodf_norm* nm) {
  if (!nm) return;
  if (nm->d_consts) {
    OnDevice on(nm->device);
    cudaFree(nm->d_consts);
  }
  delete nm;
}

int iodf_norm_forward(iodf_norm* nm, int rows, const void* r, const iodf_view* r_view, const void* b, size_t ldb,
                      const uint8_t* gate, size_t ldg, void* r_out, const iodf_view* out_view, void* n, size_t ldn,
                      void* cuda_stream) {
  if (!nm || rows < 0) return IODF_EINVAL;
  if (rows == 0) return IODF_OK;
  NormArgs a = nm->args;
  const uint32_t C = (uint32_t)a.channels;
  const size_t big = (size_t)1 << 40;
  if (!r || !r_view || !good_view(*r_view, C) || !aligned(r, a.res_i16 ? 2 : 4)) return IODF_EINVAL;
  if ((b != nullptr) != (a.has_block != 0) || (r_out != nullptr) != (a.has_block != 0) || (n != nullptr) != (a.pre != 0))
    return IODF_EINVAL;
  if (!a.has_block && gate) return IODF_EINVAL;
  if (a.has_block) {
    if (!out_view || !good_view(*out_view, C) || !aligned(r_out, a.res_i16 ? 2 : 4)) return IODF_EINVAL;
    if (!apart(*out_view, (uint64_t)rows, C)) return IODF_EINVAL;
    if (r_out == r && std::memcmp(r_view, out_view, sizeof(iodf_view))) return IODF_EINVAL;
    if (ldb < C || ldb >= big || !aligned(b, a.block_i8 ? 1 : 4)) return IODF_EINVAL;
    if (gate && ldg && (ldg < C || ldg >= big)) return IODF_EINVAL;
    a.ov = view_args(*out_view);
  }
  if (n && (ldn < C || ldn >= big)) return IODF_EINVAL;
  a.r = r;
  a.rv = view_args(*r_view);
  a.r_out = r_out;
  a.b = b;
  a.ldb = (long long)ldb;
  a.gate = gate;
  a.ldg = (long long)ldg;
  a.n = n;
  a.ldn = (long long)ldn;
  a.rows = rows;
  OnDevice on(nm->device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  return status_of(launch_norm(a, (cudaStream_t)cuda_stream));
}

}  // extern "C"

namespace iodf {

int refinement_create(const iodf_refinement& p, int device, uint64_t channels, uint64_t pixels, uint32_t max_batch, uint32_t* status,
                      Refinement* out) {
  if (!p.first || !p.up || !p.down || !p.last) return IODF_EINVAL;
  const NormArgs &f = p.first->args, &l = p.last->args;
  const ProjArgs &u = p.up->args, &d = p.down->args;
  if (p.first->device != device || p.last->device != device || p.up->device != device || p.down->device != device) return IODF_EINVAL;
  if ((uint64_t)f.channels != channels || (uint64_t)l.channels != channels || (uint64_t)u.k != channels || (uint64_t)d.n != channels || d.k != u.n)
    return IODF_EINVAL;
  if (f.res_i16 || l.res_i16 || f.has_block || !f.pre || !l.has_block || l.pre) return IODF_EINVAL;
  if ((f.n_type == IODF_U8) != (u.x_unsigned != 0) || u.y_type == IODF_I32 || (u.y_type == IODF_U8) != (d.x_unsigned != 0)) return IODF_EINVAL;
  if (d.y_type != (l.block_i8 ? IODF_I8 : IODF_I32)) return IODF_EINVAL;
  const uint64_t rows = pixels * max_batch;
  if (rows < 1 || rows > p.up->max_rows || rows > p.down->max_rows || channels > kMaxPlanes) return IODF_EINVAL;
  Refinement r;
  r.parts = p;
  r.channels = channels;
  r.pixels = pixels;
  r.status = status;
  r.ldn = up_to(channels, 16);
  r.ldu = up_to((size_t)u.n, 16);
  r.ldb = up_to(channels, 16);
  std::vector<int32_t> start;
  try {
    start.resize((size_t)max_batch + 1);
  } catch (const std::exception&) {
    return IODF_ENOMEM;
  }
  for (size_t i = 0; i < start.size(); ++i) start[i] = (int32_t)(i * pixels);
  const size_t rank = std::max<size_t>(u.max_adapters ? u.rp : 0, d.max_adapters ? d.rp : 0);
  const size_t on = 0, ou = on + up_to(rows * r.ldn, 256), ob = ou + up_to(rows * r.ldu, 256), oh = ob + up_to(rows * r.ldb * (size_t)d.y_bytes, 256),
               oq = oh + up_to(rows * rank, 256), os = oq + up_to(4 * rows, 256);
  OnDevice dev(device);
  if (dev.error() != cudaSuccess) return IODF_ECUDA;
  cudaError_t e = cudaMalloc(&r.mem, os + 4 * start.size());
  if (e != cudaSuccess) return status_of(e);
  uint8_t* m = static_cast<uint8_t*>(r.mem);
  r.n = m + on;
  r.u = m + ou;
  r.b = m + ob;
  r.h = reinterpret_cast<int8_t*>(m + oh);
  r.row_slot = reinterpret_cast<int*>(m + oq);
  r.start = reinterpret_cast<int32_t*>(m + os);
  e = cudaMemcpy(r.start, start.data(), 4 * start.size(), cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaStreamSynchronize(0);        // as in create_proj
  if (e != cudaSuccess) {
    cudaFree(r.mem);
    return status_of(e);
  }
  *out = r;
  return IODF_OK;
}

void refinement_free(Refinement* r) {
  if (r->mem) cudaFree(r->mem);
  *r = Refinement();
}

int refinement_run(const Refinement& r, int32_t* mu, uint64_t image_stride, int batch, void* stream) {
  if (!r.mem) return IODF_OK;
  const iodf_refinement& p = r.parts;
  const int rows = (int)(r.pixels * (uint64_t)batch);
  const iodf_view v{r.pixels, image_stride, r.pixels, 1};
  auto project = [&](const iodf_proj* proj, const void* x, size_t ldx, void* y, size_t ldy) {
    const bool adapters = p.image_adapter && proj->max_adapters;
    ProjArgs a = proj->args;
    a.h = r.h;
    a.row_slot = r.row_slot;
    a.status = r.status;
    return proj_forward(*proj, a, x, ldx, rows, adapters ? r.start : nullptr, adapters ? p.image_adapter : nullptr, adapters ? batch : 0, y, ldy,
                        (cudaStream_t)stream);
  };
  int rc = iodf_norm_forward(p.first, rows, mu, &v, nullptr, 0, nullptr, 0, nullptr, nullptr, r.n, r.ldn, stream);
  if (rc == IODF_OK) rc = project(p.up, r.n, r.ldn, r.u, r.ldu);
  if (rc == IODF_OK) rc = project(p.down, r.u, r.ldu, r.b, r.ldb);
  if (rc == IODF_OK) rc = iodf_norm_forward(p.last, rows, mu, &v, r.b, r.ldb, p.gate, 0, mu, &v, nullptr, 0, stream);
  return rc;
}

}  // namespace iodf
