// Error reporting shared by the C-ABI files (api.cpp, api_sequence.cpp).
#pragma once

#include <hip/hip_runtime_api.h>

#include "fdc.h"

namespace fdc {

// Records the text of fdc_last_error() for this thread and returns st.
__attribute__((format(printf, 2, 3))) fdc_status fail(fdc_status st, const char *fmt, ...);
fdc_status check_hip(hipError_t e, const char *what);

}  // namespace fdc
