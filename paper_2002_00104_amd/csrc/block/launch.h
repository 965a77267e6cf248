// What the host checks (calls.h) hand to the launches (pack.hip, norm.hip, adapter.hip).  A launch is given arguments that
// have been checked: it chooses a kernel and a grid and starts it; the caller asks the runtime for errors.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../../include/pwlq.h"
#include "../../../include/pwlq_block.h"

#define PWLQ_INTERNAL __attribute__((visibility("hidden")))

namespace pwlq_block {

inline int type_size(int type) { return type == PWLQ_F32 ? 4 : type == PWLQ_I8 ? 1 : 2; }

// Rows that one launch walks through with a workgroup each: enough to fill the chip many times over, and few enough that
// the runtime's limit of 2^32 threads is far.
inline unsigned row_grid(int64_t T, int64_t most = 1 << 20) { return (unsigned)(T < most ? T : most); }

PWLQ_INTERNAL void pack_rows(const pwlq_rows &x, int64_t T, int K, int8_t *codes, float *step, hipStream_t stream);
PWLQ_INTERNAL void unpack_rows(const int8_t *codes, const float *step, int64_t T, int K, const pwlq_rows &out, hipStream_t stream);

PWLQ_INTERNAL void norm_block(const pwlq_norm_args &a, hipStream_t stream);
PWLQ_INTERNAL size_t norm_backward_workspace(int64_t T, int64_t D, int64_t gate_rows);
PWLQ_INTERNAL void norm_backward(const pwlq_norm_backward_args &a, void *workspace, hipStream_t stream);

PWLQ_INTERNAL size_t adapter_workspace(int64_t T, int64_t K, int R);
PWLQ_INTERNAL void adapter_forward(const pwlq_adapter_args &a, void *workspace, hipStream_t stream);
PWLQ_INTERNAL size_t adapter_backward_workspace(int64_t T, int64_t K, int64_t N, int R, int adapters);
PWLQ_INTERNAL void adapter_backward(const pwlq_adapter_backward_args &a, void *workspace, hipStream_t stream);

} // namespace pwlq_block
