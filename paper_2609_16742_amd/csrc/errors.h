// The C ABI's error report, shared by its source files.
#pragma once
#include "../../include/ctc.h"

namespace ctc {
// Keeps `message` as the calling thread's ctc_last_error() and returns s.
ctc_status report(ctc_status s, const char *message);
}  // namespace ctc
