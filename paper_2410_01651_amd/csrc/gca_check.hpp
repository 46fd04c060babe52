// Argument checks shared by the files of the C ABI (api.cpp, cache_api.cpp): each keeps its
// message as the calling thread's gca_last_error().  Defined in api.cpp.
#pragma once

#include <string>

#include "gca.h"

namespace gca {

gca_status fail(gca_status s, const std::string& msg);
// The status of a launch; a failure's message names the kernel.
gca_status from_hip(hipError_t e, const char* what);
gca_status check_ptr(const void* ptr, const char* name, bool required, unsigned align);
gca_status check_ws(void* ws, size_t have, size_t need);

}  // namespace gca

#define GCA_TRY(expr)               \
  do {                              \
    const gca_status st_ = (expr);  \
    if (st_ != GCA_OK) return st_;  \
  } while (0)
