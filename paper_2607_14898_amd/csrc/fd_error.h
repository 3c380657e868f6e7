// Error reporting shared by the host files behind include/flashdecoder.h.
#pragma once

#include "../../include/flashdecoder.h"

namespace fd {
// Sets the calling thread's fd_last_error() message and returns st.
fd_status fail(fd_status st, const char* fmt, ...);
}  // namespace fd
