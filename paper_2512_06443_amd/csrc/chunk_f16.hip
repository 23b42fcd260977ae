// The kernels of the attention of chunks over a cache of type f16, outputs of that type: a translation unit of its own for the time it takes to compile.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "vlut.h"

#include "chunk_params.h"
#include "common.hip.h"
#include "launch.hip.h"
#include "chunk_kernel.hip.h"
#include "chunk_launch.hip.h"

int vlut_chunk::launch_f16(const ChunkPlan& a, const ChunkParams& p, hipStream_t stream) { return launch_chunks<_Float16, _Float16>(a, p, stream); }
