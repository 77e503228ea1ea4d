// Errors of the token-sequence operators' C ABI.
#include <stdarg.h>
#include <stdio.h>

#include "seq_common.h"

namespace dendsn_seq {

namespace {
thread_local char g_error[256] = "";
}

dendsn_status fail(dendsn_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_error, sizeof(g_error), fmt, ap);
  va_end(ap);
  return st;
}

void clear_error() { g_error[0] = 0; }

dendsn_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(DENDSN_E_HIP, "%s launch: %s", what, hipGetErrorString(e));
  return DENDSN_OK;
}

dendsn_status check_workspace(const void* ws, size_t have, size_t need, const char* query) {
  if (need == 0) return DENDSN_OK;
  if (!ws) return fail(DENDSN_E_WORKSPACE, "workspace is NULL");
  if (!aligned(ws, 16)) return fail(DENDSN_E_WORKSPACE, "workspace must be 16-byte aligned");
  if (have < need)
    return fail(DENDSN_E_WORKSPACE, "workspace of %zu bytes is smaller than %s() = %zu", have, query, need);
  return DENDSN_OK;
}

}  // namespace dendsn_seq

extern "C" const char* dendsn_seq_last_error(void) { return dendsn_seq::g_error; }
