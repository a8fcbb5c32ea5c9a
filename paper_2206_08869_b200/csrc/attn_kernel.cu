// Attention over the cache of blocks (include/iodf.h: iodf_attn_forward): which kernel takes a call.
#include "attn.h"

#include <algorithm>

#include "attn_kernels.h"

namespace iodf {

namespace {

// Both kernels' times as the host can tell them, in ns: contexts as long as the table is wide, rows spread evenly over the requests. Units are
// of `cols` rows and a head of the cache: whole ones and one that is not for each request at most, or those of each token by itself.
long long blocks_of(const AttnArgs& a, const ForwardArgs& f) { return a.window ? std::min<long long>(f.width, a.window / kAttnBlock + 2) : f.width; }
long long units_of(const AttnArgs& a, const ForwardArgs& f, int cols) {
  return std::min((long long)f.rows * a.group / cols + f.n, (long long)f.rows * ((a.group + cols - 1) / cols)) * a.kv;
}
// us measured (and by this), 8 heads of 128, contexts of 4096 tokens, 8, 16, 32, 64, 128 rows of a request: 1 request 19 25 25 32 56 (15 16 19 25 38),
// 16 requests 55 85 126 210 406 (44 62 111 210 406), 64 requests 127 215 409 774 1526 (136 210 406 800 1586)
long long split_ns(const AttnArgs& a, const ForwardArgs& f) {
  const int cols = attn_split_cols(a, f);
  return 13000 + units_of(a, f, cols) * blocks_of(a, f) * (cols > 8 ? 120 : 75) / 10;
}
// ... 1, 16, 64 requests 73, 78, 269 (75, 75, 267), with contexts of 512 tokens 20, 21, 56 (22, 22, 54), whatever the rows up to 128
long long tile_ns(const AttnArgs& a, const ForwardArgs& f) {
  return 11500 + (units_of(a, f, 128) + a.sms - 1) / a.sms * (3000 + 1900 * blocks_of(a, f));
}

}  // namespace

cudaError_t configure_attn_kernels(int device, AttnArgs* a) {
  cudaError_t e = cudaDeviceGetAttribute(&a->sms, cudaDevAttrMultiProcessorCount, device);
  if (e == cudaSuccess) e = configure_attn_cache();
  if (e == cudaSuccess) e = configure_attn_split(a);
  return e == cudaSuccess ? configure_attn_tile() : e;
}

cudaError_t launch_attn_forward(const AttnArgs& a, const CacheArgs& c, const ForwardArgs& f, const CUtensorMap& k_map, const CUtensorMap& v_map,
                                cudaStream_t stream) {
  return f.n <= kAttnSplitRequests && split_ns(a, f) <= tile_ns(a, f) ? launch_attn_split(a, c, f, k_map, v_map, stream)
                                                                       : launch_attn_tile(a, c, f, k_map, v_map, stream);
}

}  // namespace iodf
