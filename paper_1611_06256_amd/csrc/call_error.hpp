// Error text of the calls that are not the scheduler's: thread-local, read through ga3c_last_error().  Defined in ga3c.hip.
#pragma once

namespace ga3c {
int call_fail(int code, const char *fmt, ...);      // stores the text, returns code
}  // namespace ga3c
