// What the library's translation units share on the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dqrm_host {

// keeps the text for dqrm_last_hip_error() and returns DQRM_ERR_HIP
__attribute__((visibility("hidden"))) int32_t hip_fail(hipError_t e, const char *what);

} // namespace dqrm_host
