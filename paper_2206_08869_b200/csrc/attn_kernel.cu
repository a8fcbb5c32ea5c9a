// Attention over the cache of blocks (include/iodf.h: iodf_attn_forward): which kernel takes a call.
#include "attn.h"

#include <algorithm>

#include "attn_kernels.h"

namespace iodf {

namespace {

// Both kernels' times as the host can tell them, in ns: contexts as long as the table is wide, rows spread evenly over the requests. Units are
// of `cols` rows and a head of the cache, or fewer where a request's or a token's rows end. Of 60 sizes measured with both (1, 16 and 64
// requests of 8 to 128 rows, contexts of 512 and 4096 tokens, 8 heads of 128 and 4 of 64) the slower one is taken for five, which
// take 1.1 to 1.25 times as long as they could.
long long blocks_of(const AttnArgs& a, const ForwardArgs& f) { return a.window ? std::min<long long>(f.width, a.window / kAttnBlock + 2) : f.width; }
long long units_of(const AttnArgs& a, const ForwardArgs& f, int cols) {
  const long long flat = ((long long)f.rows * a.group + f.n - 1) / f.n;
  return std::min((flat + cols - 1) / cols * f.n, (long long)f.rows * ((a.group + cols - 1) / cols)) * a.kv;
}
// us measured (and by this), 8 heads of 128, contexts of 4096 tokens, 8, 16, 32, 64, 128 rows of a request: 1 request 18 25 25 32 56 (15 16 19 25 38),
// 16 requests 53 84 125 207 398 (44 62 111 210 406), 64 requests 125 213 403 763 1498 (136 210 406 799 1586)
long long split_ns(const AttnArgs& a, const ForwardArgs& f) {
  const int cols = attn_split_cols(a, f);
  return 13000 + units_of(a, f, cols) * blocks_of(a, f) * (cols > 8 ? 120 : 75) / 10;
}
// ... 1, 16, 64 requests 69, 76, 262 (75, 75, 267), with contexts of 512 tokens 20, 21, 57 (22, 22, 54), whatever the rows up to 128
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
