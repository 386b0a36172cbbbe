// libasd: the tensor-core attention kernel's host side (asd_attention_tc.cu),
// for the entry point in asd_attention.cu.
#pragma once

#include <cuda_runtime.h>

#include "asd.h"
#include "asd_attention.cuh"

namespace asd_detail {

// Whether the kernel takes this call's types, head width, strides and alignment.
bool attention_tc_takes(const asd_kv_cache* cache, const AttnParams& p);
size_t attention_tc_bytes(const asd_kv_cache* cache, int T, int q_heads);
int launch_attention_tc(const asd_kv_cache* cache, AttnParams p, char* workspace, cudaStream_t stream);

}  // namespace asd_detail
