// What a C entry point returns: a status code, with the text that
// bnn_last_error() gives for it on this thread.  Defined in api.cpp.
#pragma once

#include <hip/hip_runtime_api.h>

#include "bnn.h"

namespace bnn {

// Sets the thread's error text (printf form) and returns st.
bnn_status fail(bnn_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Clears the thread's error text and returns BNN_OK.
bnn_status ok();
// ok(), or BNN_ERR_HIP with the runtime's text for e.
bnn_status hip_status(hipError_t e, const char* where);

}  // namespace bnn
