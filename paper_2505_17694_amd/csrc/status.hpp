// Failures of HIP calls, kept for codec_last_error_message.
#pragma once

namespace codec {

// Records which HIP call failed and why (`code`, a hipError_t value); returns CODEC_ERR_HIP.
int hip_failure(const char *what, int code);

}  // namespace codec
