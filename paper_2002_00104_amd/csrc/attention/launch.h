// What the host checks (calls.h) hand to the launches (append.hip, attend.hip).  A launch is given arguments that have
// been checked: it chooses a kernel and a grid and starts it; the caller asks the runtime for errors.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../../include/pwlq.h"
#include "../../../include/pwlq_attention.h"

#define PWLQ_INTERNAL __attribute__((visibility("hidden")))

namespace pwlq_attention {

PWLQ_INTERNAL void append(const pwlq_append_args &a, hipStream_t stream);
PWLQ_INTERNAL void read(const pwlq_read_args &a, hipStream_t stream);

PWLQ_INTERNAL size_t attend_workspace(const pwlq_attend_args &a);
PWLQ_INTERNAL void attend(const pwlq_attend_args &a, void *workspace, hipStream_t stream);

} // namespace pwlq_attention
