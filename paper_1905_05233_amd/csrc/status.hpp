// Statuses of the C ABI: every failure is a wg_status and a message of the
// calling thread (api.hip), which winograd_last_error reads.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "winograd_crt.h"

namespace wg {

wg_status fail(wg_status s, const std::string& msg);
wg_status from_hip(hipError_t e, const char* what);   // WG_OK for hipSuccess

}  // namespace wg
