// Low-rank adapters of many requests (adapters.hip) as the C entry points see them.
#pragma once

#include "hawk_internal.h"

namespace hawk {

size_t adapter_plan_bytes(int rows, int n_adapters);
int launch_adapter_plan(const int32_t* row_start, const int32_t* adapter, int n_seq, int rows, int n_adapters, void* plan, size_t plan_bytes,
                        hipStream_t stream);
int launch_adapter_apply(const hawk_adapters* w, const void* plan, size_t plan_bytes, int rows, const hawk_matrix* x, const hawk_matrix* base,
                         const hawk_matrix* out, void* workspace, size_t workspace_bytes, hipStream_t stream);
size_t adapter_apply_workspace_bytes(const hawk_adapters* w, int rows);

}  // namespace hawk
