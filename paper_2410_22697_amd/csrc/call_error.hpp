// call_error.hpp - the message that massive_last_error(NULL) gives, for calls
// that have no context.
#pragma once

namespace ms {
// Keeps the message on this thread and returns the code. Never throws.
__attribute__((visibility("hidden"), format(printf, 2, 3))) int call_error(int code, const char* fmt, ...) noexcept;
}  // namespace ms
