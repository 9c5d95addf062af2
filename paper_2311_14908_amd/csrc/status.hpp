// status.hpp -- what the files of the C ABI share on the host: the thread's error message, the check
// of a call's options, and the failure of a HIP call.
#pragma once

#include <hip/hip_runtime.h>

#include "svmx.h"

namespace svmx {

// The thread's message; returns st.
svm_status fail(svm_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();
// Options of a call that takes only their stream (o may be NULL); false where they are malformed.
bool stream_of(const svm_options *o, hipStream_t *s);

#define HIPCHK(expr)                                                                      \
  do {                                                                                    \
    hipError_t e_ = (expr);                                                               \
    if (e_ != hipSuccess) return fail(SVM_EDEVICE, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

}  // namespace svmx
