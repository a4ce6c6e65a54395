// The status word of the scoring kernels (logprobs.hip, joint_logprobs.hip) on the
// current device; end_status_take reads it with its own for fusion_device_status.
#pragma once

#include <cstdint>

namespace fusion {
int score_status_word(int32_t **word);
}  // namespace fusion
