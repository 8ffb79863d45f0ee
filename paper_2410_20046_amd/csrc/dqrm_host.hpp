// What the library's translation units share on the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dqrm_host {

// keeps the text for dqrm_last_hip_error() and returns DQRM_ERR_HIP
__attribute__((visibility("hidden"))) int32_t hip_fail(hipError_t e, const char *what);

// Softmax cross entropy: joins the tiles' parts of each row (maximum and sum of powers of two, [tiles][rows] pairs of floats) to lse and loss
// from the target's logit `at`.  Lies with the status word, where a target past the last class is recorded.
__attribute__((visibility("hidden"))) void launch_xent_join(const void *parts, int64_t tiles, int64_t rows, const float *at, const int64_t *targets,
                                                            int64_t classes, float *loss, float *lse, hipStream_t st);

} // namespace dqrm_host
