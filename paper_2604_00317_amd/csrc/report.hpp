// Error reports of the C entry points: the message goes to nimble_last_error of this thread.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/nimble_plan.h"

namespace nimble {

void report_clear() noexcept;
nimble_status_t report(nimble_status_t status, const char *message) noexcept;
nimble_status_t report_hip(hipError_t e, const char *what) noexcept;

}  // namespace nimble
