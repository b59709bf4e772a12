// What the C entry points share: the plan handle, the per-thread error record
// and the checks before a launch.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "../../include/ccl.h"
#include "host/plan.hpp"

struct ccl_plan_s {
  ccl::Plan plan;
};

namespace ccl {
namespace api {

// Record an error (or none) of the calling thread and return its status.
ccl_status fail(ccl_status s, const std::string& msg);
ccl_status ok();
ccl_status from(Status s, const std::string& msg);
ccl_status hip_status(hipError_t e, const char* what);
// The current device is a gfx950.
ccl_status check_device();

inline bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned(p, 16); }

bool addressing_in_bounds(const Plan& p, const OperandAddr& a, const OperandAddr& b, const OperandAddr& c,
                          int64_t a_bytes, int64_t b_bytes, int64_t c_bytes);
bool offsets_fit(const Plan& p, const OperandAddr& a, const OperandAddr& b);

}  // namespace api
}  // namespace ccl
