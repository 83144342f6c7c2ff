// The message behind hpf_last_error, shared by the files that define entry points of the C ABI.
#pragma once
#include "../../include/hpf.h"

namespace hpf {

// Records the message for this thread and returns st.
hpf_status fail(hpf_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace hpf
