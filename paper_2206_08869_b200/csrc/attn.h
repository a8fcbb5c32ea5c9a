// Integer attention over a cache of blocks (include/iodf.h: iodf_attn_*): launch arguments.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace iodf {

constexpr int kAttnBlock = 128;          // tokens of a block
constexpr int kAttnMaxBlocks = 1024;     // of a request: sums of 131072 products of at most 128 * 127 fit 32 bits
constexpr int kAttnMaxRequests = 16384;  // of a call of iodf_attn_plan: their prefix sums lie in shared memory
constexpr int kAttnSplitRequests = 8192; // of a call that the kernel for few rows takes: so do its prefix sums
constexpr int kAttnMaxTeam = 16;
constexpr int kAttnMaxExp = 12;          // exponents above count as this
constexpr int kRotaryHalf = 1, kRotaryInterleaved = 2;

struct AttnArgs {                        // what a handle holds
  int heads, kv, group, dim;             // group = heads / kv
  int x_i8;
  int rot, layout, positions;
  const short2* rotary;                  // [positions][rot / 2] cos, sin in 2^-14
  int k_headroom, v_headroom;            // eighths
  uint32_t score_m0;
  int score_s;
  int causal, window;
  int y_type, y_bytes, lo, hi;
  int y_full;                            // 8-bit signed outputs, clipped to their type's range
  const int4* out;                       // [heads * dim] {M0, s, low and high word of 2^(30 + s)}
  uint32_t* status;                      // [0] a bounded wait gave up, [1] requests or rows that could not be served
  int sms;
  int clusters[kAttnMaxTeam + 1];        // of the kernel for few rows: clusters of 8 .. 16 CTAs that run at once
};

struct CacheArgs {
  int8_t *k, *v;                         // [blocks][kv][128][dim], [blocks][kv][dim][128]
  uint8_t *k_exp, *v_exp;                // [blocks][kv]
  int blocks;
};

struct PlanArgs {
  int n, rows, width, ring_size;
  long long ldt;
  const int32_t *held, *add, *state;
  int32_t *table, *ring, *held_out, *row_start, *slot, *position, *state_out;
  uint32_t* status;
};

struct AppendArgs {
  const void *q, *k, *v;
  long long ldq, ldk, ldv;
  int rows;
  const int32_t *slot, *position;
  int8_t* q8;
  uint8_t* q_exp;
  int vector;                            // a lane's elements can be read at once
};

struct ForwardArgs {
  const int8_t* q8;
  const uint8_t* q_exp;
  const int32_t *row_start, *held, *table;
  long long ldt, ldy;
  int rows, n, width;
  void* y;
  int vector;                            // four neighbouring outputs lie on a boundary of their size
};

cudaError_t configure_attn_kernels(int device, AttnArgs* a);      // on the current device, before the first launch
cudaError_t launch_attn_plan(const PlanArgs& p, int sms, cudaStream_t stream);
cudaError_t launch_attn_append(const AttnArgs& a, const CacheArgs& c, const AppendArgs& p, cudaStream_t stream);
// k_map, v_map: of the cache as rows of `dim` and of 128 bytes, a block's part of one head to a box, swizzled over a row's width
cudaError_t launch_attn_forward(const AttnArgs& a, const CacheArgs& c, const ForwardArgs& f, const CUtensorMap& k_map, const CUtensorMap& v_map,
                                cudaStream_t stream);

}  // namespace iodf
