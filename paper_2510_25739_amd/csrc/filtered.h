// Draws from filtered rows (filtered.hip) as the C entry points see them.
#pragma once

#include "hawk_internal.h"

namespace hawk {

size_t sample_filtered_workspace_bytes(int rows, int n);
int launch_sample_filtered(const void* logits, int dtype, int64_t row_stride, const int32_t* skip, const float* u, const float* temperature,
                           const int32_t* top_k, const float* top_p, const float* min_p, int rows, int n, int32_t* out_token, float* out_prob,
                           int32_t* out_kept, void* workspace, size_t workspace_bytes, hipStream_t stream);

}  // namespace hawk
