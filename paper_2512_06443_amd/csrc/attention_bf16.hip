// The attention's kernels over a cache of type bf16: a translation unit of its own for the time it takes to compile.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "vlut.h"

#include "attention_params.h"
#include "common.hip.h"
#include "launch.hip.h"
#include "attention_kernel.hip.h"
#include "attention_launch.hip.h"

int vlut_attention::launch_bf16(const AttendPlan& a, const AttendParams& p, hipStream_t stream) { return launch_attend<__bf16>(a, p, stream); }
