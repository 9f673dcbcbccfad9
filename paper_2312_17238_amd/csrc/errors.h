// How the library's other sources report what went wrong: into the calling thread's moe_last_error / moe_last_hip_error.
#pragma once
#include <stdint.h>

namespace moe {

// Keeps `text` (and `hip_err` unless 0) for the calling thread and returns `code`.
__attribute__((visibility("hidden"))) int32_t report_error(int32_t code, int32_t hip_err, const char *text);

}  // namespace moe
