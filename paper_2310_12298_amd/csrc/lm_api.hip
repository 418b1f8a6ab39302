// Errors of the calls of jorge_lm.h.
#include "lm_common.hpp"

#include <stdio.h>

namespace jorge_lm {
namespace {
thread_local char g_error[256] = "";
}

jorge_status refuse(jorge_status st, const char* why) {
    snprintf(g_error, sizeof g_error, "%s", why);
    return st;
}

jorge_status launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return JORGE_OK;
    snprintf(g_error, sizeof g_error, "%s: %s", what, hipGetErrorString(e));
    return JORGE_ERR_HIP;
}
}  // namespace jorge_lm

extern "C" const char* jorge_lm_last_error(void) { return jorge_lm::g_error; }
