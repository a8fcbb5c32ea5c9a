// Attention over the cache of blocks (include/iodf.h: iodf_attn_forward): which kernel takes a call.
#include "attn.h"

#include "attn_kernels.h"

namespace iodf {

cudaError_t configure_attn_kernels(int device, AttnArgs* a) {
  cudaError_t e = cudaDeviceGetAttribute(&a->sms, cudaDevAttrMultiProcessorCount, device);
  if (e == cudaSuccess) e = configure_attn_cache();
  if (e == cudaSuccess) e = configure_attn_split(a);
  return e == cudaSuccess ? configure_attn_tile() : e;
}

cudaError_t launch_attn_forward(const AttnArgs& a, const CacheArgs& c, const ForwardArgs& f, const CUtensorMap& k_map, const CUtensorMap& v_map,
                                cudaStream_t stream) {
  const long long flat = (long long)f.rows * a.group;
  if (flat <= 32ll * f.n && f.n <= kAttnSplitRequests) return launch_attn_split(a, c, f, k_map, v_map, stream);
  return launch_attn_tile(a, c, f, k_map, v_map, stream);
}

}  // namespace iodf
