// Status bits of the scoring kernels (logprobs.hip, joint_logprobs.hip), taken and
// cleared; end_status_take hands them on to fusion_device_status with its own.
#pragma once

#include <cstdint>

namespace fusion {
int score_status_take(int32_t *bits);
int joint_score_status_take(int32_t *bits);
}  // namespace fusion
