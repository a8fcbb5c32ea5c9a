// The kernels behind launch_attn_forward, and what each needs on a device before its first launch.
#pragma once
#include "attn.h"

namespace iodf {

cudaError_t configure_attn_cache();
cudaError_t configure_attn_tile();
cudaError_t launch_attn_tile(const AttnArgs& a, const CacheArgs& c, const ForwardArgs& f, const CUtensorMap& k_map, const CUtensorMap& v_map,
                             cudaStream_t stream);
cudaError_t configure_attn_split(AttnArgs* a);
int attn_split_cols(const AttnArgs& a, const ForwardArgs& f);      // rows of a unit of the kernel for few rows
cudaError_t launch_attn_split(const AttnArgs& a, const CacheArgs& c, const ForwardArgs& f, const CUtensorMap& k_map, const CUtensorMap& v_map,
                              cudaStream_t stream);

}  // namespace iodf
