// C ABI of integer attention over a cache of blocks (include/iodf.h). Host side only: checks, device buffers, launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <exception>
#include <new>
#include <vector>

#include "../../include/iodf.h"
#include "api_common.h"
#include "attn.h"

using namespace iodf;

struct iodf_attn {
  int device = 0;
  EncodeTiled encode = nullptr;
  AttnArgs args{};
  void* d_mem = nullptr;                     // rotary table, constants of the outputs, status words
};

namespace {

constexpr uint32_t kMaxHeads = 1024, kMaxGroup = 128, kMaxPositions = 1u << 24;
constexpr size_t kMaxStride = (size_t)1 << 40;

int create_attn(const iodf_attn_desc& d, int device, iodf_attn& h) {
  if (d.heads < 1 || d.kv_heads < 1 || d.heads % d.kv_heads) return IODF_EINVAL;
  if (d.head_dim < 1) return IODF_EINVAL;
  if (d.head_dim != 32 && d.head_dim != 64 && d.head_dim != 128) return IODF_EUNSUPPORTED;
  if (d.heads > kMaxHeads || d.heads / d.kv_heads > kMaxGroup) return IODF_EUNSUPPORTED;
  if (d.x_type != IODF_I8 && d.x_type != IODF_I32) return IODF_EINVAL;
  if (d.rotary_dim) {
    if (d.rotary_dim > d.head_dim || d.rotary_dim % 2 || !d.rotary || d.positions < 1) return IODF_EINVAL;
    if (d.rotary_layout != IODF_ROTARY_HALF && d.rotary_layout != IODF_ROTARY_INTERLEAVED) return IODF_EINVAL;
    if (d.rotary_dim % 16 || d.positions > kMaxPositions) return IODF_EUNSUPPORTED;
    for (size_t i = 0; i < (size_t)d.positions * d.rotary_dim; ++i)
      if (d.rotary[i] < -16384 || d.rotary[i] > 16384) return IODF_EINVAL;
  }
  if (d.k_headroom > 8 || d.v_headroom > 8) return IODF_EINVAL;
  if (d.score_m0 < (1 << 30) || d.score_s < 0 || d.score_s > 62) return IODF_EINVAL;
  if (d.causal > 1 || d.window > (1u << 30)) return IODF_EINVAL;
  if (d.y_type != IODF_I8 && d.y_type != IODF_U8 && d.y_type != IODF_I32) return IODF_EINVAL;
  int lo = INT32_MIN, hi = INT32_MAX;
  if (d.has_clamp) {
    if (d.clamp_lo > d.clamp_hi) return IODF_EINVAL;
    lo = d.clamp_lo;
    hi = d.clamp_hi;
  }
  if (d.y_type == IODF_I8 && (lo < -128 || hi > 127)) return IODF_EINVAL;
  if (d.y_type == IODF_U8 && (lo < 0 || hi > 255)) return IODF_EINVAL;
  const size_t N = (size_t)d.heads * d.head_dim, R = (size_t)d.positions * (d.rotary_dim / 2);
  if (!d.out_m0 || !d.out_s) return IODF_EINVAL;
  std::vector<int4> out(N);
  for (size_t n = 0; n < N; ++n) {
    if (d.out_m0[n] < (1 << 30) || d.out_s[n] < 0 || d.out_s[n] > 31) return IODF_EINVAL;
    const uint64_t add = 1ull << (30 + d.out_s[n]);
    out[n] = make_int4(d.out_m0[n], d.out_s[n], (int)(uint32_t)add, (int)(uint32_t)(add >> 32));
  }
  h.device = device;
  OnDevice on(device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  h.encode = tensor_map_encoder();
  if (!h.encode) return IODF_ECUDA;
  cudaError_t e = configure_attn_kernels(device, &h.args);
  const size_t o_out = up_to(4 * R, 256), o_status = o_out + up_to(16 * N, 256);
  if (e == cudaSuccess) e = cudaMalloc(&h.d_mem, o_status + 8);
  if (e != cudaSuccess) return status_of(e);
  uint8_t* m = static_cast<uint8_t*>(h.d_mem);
  if (R) e = cudaMemcpy(m, d.rotary, 4 * R, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaMemcpy(m + o_out, out.data(), 16 * N, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaMemset(m + o_status, 0, 8);
  // A copy from pageable memory is only known to have left it: the first call may be on a stream that does not wait for the rest.
  if (e == cudaSuccess) e = cudaStreamSynchronize(0);
  if (e != cudaSuccess) return status_of(e);
  AttnArgs& a = h.args;
  a.heads = (int)d.heads;
  a.kv = (int)d.kv_heads;
  a.group = (int)(d.heads / d.kv_heads);
  a.dim = (int)d.head_dim;
  a.x_i8 = d.x_type == IODF_I8;
  a.rot = (int)d.rotary_dim;
  a.layout = d.rotary_dim ? (int)d.rotary_layout : (int)IODF_ROTARY_HALF;
  a.positions = d.rotary_dim ? (int)d.positions : 1;
  a.rotary = reinterpret_cast<const short2*>(m);
  a.k_headroom = (int)d.k_headroom;
  a.v_headroom = (int)d.v_headroom;
  a.score_m0 = (uint32_t)d.score_m0;
  a.score_s = d.score_s;
  a.causal = (int)d.causal;
  a.window = (int)d.window;
  a.y_type = (int)d.y_type;
  a.y_bytes = d.y_type == IODF_I32 ? 4 : 1;
  a.y_full = d.y_type == IODF_I8 && lo == -128 && hi == 127;
  a.lo = lo;
  a.hi = hi;
  a.out = reinterpret_cast<const int4*>(m + o_out);
  a.status = reinterpret_cast<uint32_t*>(m + o_status);
  return IODF_OK;
}

struct Span {                                 // an operand's bytes, from its first to behind its last one
  uintptr_t begin, end;
  Span(const void* p, size_t bytes) : begin(reinterpret_cast<uintptr_t>(p)), end(begin + bytes) {}
  bool meets(const Span& o) const { return begin < o.end && o.begin < end && begin < end && o.begin < o.end; }
};

size_t extent(size_t rows, size_t stride, size_t width, size_t bytes) { return rows ? ((rows - 1) * stride + width) * bytes : 0; }

// Does any of `out` overlap another of `out` or any of `in`?
template <size_t N, size_t M>
bool overlap(const Span (&out)[N], const Span (&in)[M]) {
  for (size_t i = 0; i < N; ++i) {
    for (size_t j = i + 1; j < N; ++j)
      if (out[i].meets(out[j])) return true;
    for (size_t j = 0; j < M; ++j)
      if (out[i].meets(in[j])) return true;
  }
  return false;
}

// Blocks of a cache or a ring, times the heads of a block: a slot, and a row of the cache's tensor maps, is a 32-bit number.
constexpr uint64_t kMostBlocks = (uint64_t)INT32_MAX / kAttnBlock;

// The cache's pointers and sizes: 8-bit rows are read in tiles of 16-byte pieces.
int check_cache(const iodf_attn& h, const iodf_attn_cache* c) {
  if (!c || !c->k || !c->v || !c->k_exp || !c->v_exp || c->blocks < 1 || !aligned(c->k, 16) || !aligned(c->v, 16)) return IODF_EINVAL;
  return (uint64_t)c->blocks * h.args.kv > kMostBlocks ? IODF_EUNSUPPORTED : IODF_OK;
}

CacheArgs cache_args(const iodf_attn_cache& c) { return {c.k, c.v, c.k_exp, c.v_exp, (int)c.blocks}; }

size_t cache_bytes(const iodf_attn& h, const iodf_attn_cache& c) { return (size_t)c.blocks * h.args.kv * kAttnBlock * h.args.dim; }

// int8 [rows][width], boxes of box_rows rows, swizzled over a row's width (32, 64 or 128 bytes)
bool cache_map(const iodf_attn& h, const void* base, uint64_t width, uint64_t rows, uint32_t box_rows, CUtensorMap* out) {
  const cuuint64_t dims[2] = {width, rows}, strides[1] = {width};
  const cuuint32_t box[2] = {(cuuint32_t)width, box_rows}, steps[2] = {1, 1};
  const CUtensorMapSwizzle swizzle = width == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : width == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B;
  return h.encode(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

extern "C" {

int iodf_attn_create(const iodf_attn_desc* desc, int device, iodf_attn** out) {
  if (!desc || !out) return IODF_EINVAL;
  *out = nullptr;
  if (desc->abi_version != IODF_ABI_VERSION) return IODF_EVERSION;
  iodf_attn* h = new (std::nothrow) iodf_attn();
  if (!h) return IODF_ENOMEM;
  int rc;
  try {
    rc = create_attn(*desc, device, *h);
  } catch (const std::exception&) {              // out of host memory, or a size beyond what a vector may have
    rc = IODF_ENOMEM;
  }
  if (rc != IODF_OK) {
    iodf_attn_destroy(h);
    return rc;
  }
  *out = h;
  return IODF_OK;
}

void iodf_attn_destroy(iodf_attn* h) {
  if (!h) return;
  if (h->d_mem) {
    OnDevice on(h->device);
    cudaFree(h->d_mem);
  }
  delete h;
}

int iodf_attn_plan(iodf_attn* h, int n_req, const int32_t* held, const int32_t* add, int32_t* table, size_t ldt, uint32_t width, int32_t* ring,
                   uint32_t ring_size, const int32_t* state, int rows, int32_t* held_out, int32_t* row_start, int32_t* slot, int32_t* position,
                   int32_t* state_out, void* cuda_stream) {
  if (!h || n_req < 0 || rows < 0) return IODF_EINVAL;
  if (!state || !state_out || !row_start || (n_req && (!held || !add || !table || !held_out)) || (rows && (!slot || !position))) return IODF_EINVAL;
  if (!ring || ring_size < 1 || width < 1 || ldt < width || ldt >= kMaxStride) return IODF_EINVAL;
  if (n_req > kAttnMaxRequests || width > (uint32_t)kAttnMaxBlocks || ring_size > kMostBlocks || rows > (1 << 30)) return IODF_EUNSUPPORTED;
  for (const void* p : {(const void*)held, (const void*)add, (const void*)table, (const void*)ring, (const void*)state, (const void*)held_out,
                        (const void*)row_start, (const void*)slot, (const void*)position, (const void*)state_out})
    if (!aligned(p, 4)) return IODF_EINVAL;
  const size_t n = (size_t)n_req;
  const Span outs[] = {{table, 4 * extent(n, ldt, width, 1)}, {ring, 4 * (size_t)ring_size}, {held_out, 4 * n}, {row_start, 4 * (n + 1)},
                       {slot, 4 * (size_t)rows}, {position, 4 * (size_t)rows}, {state_out, 8}};
  const Span ins[] = {{held, 4 * n}, {add, 4 * n}, {state, 8}};
  if (overlap(outs, ins)) return IODF_EINVAL;     // every CTA reads what others' outputs would change
  PlanArgs p{n_req, rows, (int)width, (int)ring_size, (long long)ldt, held, add, state, table, ring, held_out, row_start, slot, position, state_out,
             h->args.status};
  OnDevice on(h->device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  return status_of(launch_attn_plan(p, h->args.sms, (cudaStream_t)cuda_stream));
}

int iodf_attn_append(iodf_attn* h, int rows, const void* q, size_t ldq, const void* k, size_t ldk, const void* v, size_t ldv, const int32_t* slot,
                     const int32_t* position, const iodf_attn_cache* cache, int8_t* q8, uint8_t* q_exp, void* cuda_stream) {
  if (!h || rows < 0) return IODF_EINVAL;
  if (const int rc = check_cache(*h, cache)) return rc;
  if (rows == 0) return IODF_OK;
  const AttnArgs& a = h->args;
  const size_t R = (size_t)rows, x = a.x_i8 ? 1 : 4, nq = (size_t)a.heads * a.dim, nk = (size_t)a.kv * a.dim;
  if (rows > (1 << 30)) return IODF_EUNSUPPORTED;
  if (!q || !k || !v || !slot || !position || !q8 || !q_exp) return IODF_EINVAL;
  if (!aligned(q, x) || !aligned(k, x) || !aligned(v, x) || !aligned(slot, 4) || !aligned(position, 4) || !aligned(q8, 16)) return IODF_EINVAL;
  if (ldq < nq || ldk < nk || ldv < nk || ldq >= kMaxStride || ldk >= kMaxStride || ldv >= kMaxStride) return IODF_EINVAL;
  const size_t blocks = (size_t)cache->blocks * a.kv;
  const Span outs[] = {{cache->k, cache_bytes(*h, *cache)}, {cache->v, cache_bytes(*h, *cache)}, {cache->k_exp, blocks}, {cache->v_exp, blocks},
                       {q8, R * nq}, {q_exp, R * a.heads}};
  const Span ins[] = {{q, extent(R, ldq, nq, x)}, {k, extent(R, ldk, nk, x)}, {v, extent(R, ldv, nk, x)}, {slot, 4 * R}, {position, 4 * R}};
  if (overlap(outs, ins)) return IODF_EINVAL;
  const size_t lane = 4 * x;                      // bytes of a lane's elements
  const bool vector = aligned(q, lane) && aligned(k, lane) && aligned(v, lane) && ldq * x % lane == 0 && ldk * x % lane == 0 && ldv * x % lane == 0;
  const AppendArgs p{q, k, v, (long long)ldq, (long long)ldk, (long long)ldv, rows, slot, position, q8, q_exp, vector};
  OnDevice on(h->device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  return status_of(launch_attn_append(a, cache_args(*cache), p, (cudaStream_t)cuda_stream));
}

int iodf_attn_forward(iodf_attn* h, int rows, const int8_t* q8, const uint8_t* q_exp, const int32_t* row_start, const int32_t* held, int n_req,
                      const int32_t* table, size_t ldt, uint32_t width, const iodf_attn_cache* cache, void* y, size_t ldy, void* cuda_stream) {
  if (!h || rows < 0 || n_req < 0) return IODF_EINVAL;
  if (const int rc = check_cache(*h, cache)) return rc;
  if (rows == 0 || n_req == 0) return IODF_OK;
  const AttnArgs& a = h->args;
  const size_t R = (size_t)rows, n = (size_t)n_req, N = (size_t)a.heads * a.dim;
  if (!q8 || !q_exp || !row_start || !held || !table || !y) return IODF_EINVAL;
  if (!aligned(q8, 16) || !aligned(row_start, 4) || !aligned(held, 4) || !aligned(table, 4) || !aligned(y, (size_t)a.y_bytes)) return IODF_EINVAL;
  if (width < 1 || ldt < width || ldt >= kMaxStride || ldy < N || ldy >= kMaxStride) return IODF_EINVAL;
  if (width > (uint32_t)kAttnMaxBlocks || rows > (1 << 30) / a.heads || n_req > (1 << 20)) return IODF_EUNSUPPORTED;
  const size_t blocks = (size_t)cache->blocks * a.kv;
  const Span outs[] = {{y, extent(R, ldy, N, (size_t)a.y_bytes)}};
  const Span ins[] = {{q8, R * N}, {q_exp, R * a.heads}, {row_start, 4 * (n + 1)}, {held, 4 * n}, {table, 4 * extent(n, ldt, width, 1)},
                      {cache->k, cache_bytes(*h, *cache)}, {cache->v, cache_bytes(*h, *cache)}, {cache->k_exp, blocks}, {cache->v_exp, blocks}};
  if (overlap(outs, ins)) return IODF_EINVAL;
  const ForwardArgs f{q8, q_exp, row_start, held, table, (long long)ldt, (long long)ldy, rows, n_req, (int)width, y,
                      ldy % 4 == 0 && aligned(y, 4 * (size_t)a.y_bytes)};
  OnDevice on(h->device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  CUtensorMap k_map, v_map;
  if (!cache_map(*h, cache->k, (uint64_t)a.dim, blocks * kAttnBlock, kAttnBlock, &k_map) ||
      !cache_map(*h, cache->v, (uint64_t)kAttnBlock, blocks * a.dim, (uint32_t)a.dim, &v_map))
    return IODF_ECUDA;
  return status_of(launch_attn_forward(a, cache_args(*cache), f, k_map, v_map, (cudaStream_t)cuda_stream));
}

int iodf_attn_check(iodf_attn* h, void* cuda_stream, uint32_t* bad) {
  if (!h) return IODF_EINVAL;
  if (bad) *bad = 0;
  OnDevice on(h->device);
  if (on.error() != cudaSuccess) return IODF_ECUDA;
  uint32_t st[2] = {0, 0};
  cudaError_t e = cudaStreamSynchronize((cudaStream_t)cuda_stream);
  if (e == cudaSuccess) e = cudaMemcpy(st, h->args.status, 8, cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && (st[0] || st[1])) e = cudaMemset(h->args.status, 0, 8);
  if (e == cudaSuccess) e = cudaStreamSynchronize(0);
  if (e != cudaSuccess) return IODF_ECUDA;
  if (bad) *bad = st[1];
  return st[0] ? IODF_ETIMEOUT : st[1] ? IODF_EDATA : IODF_OK;
}

}  // extern "C"
