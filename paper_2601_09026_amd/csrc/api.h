// What the files with exported functions share.
#pragma once
#include <hip/hip_runtime_api.h>

#include <mutex>

namespace mg {

std::recursive_mutex& call_mutex();        // taken by every entry point that enqueues work
int hip_failed(hipError_t e);              // notes the error for mgrit_last_hip_error(); MGRIT_HIP_ERROR

}  // namespace mg
