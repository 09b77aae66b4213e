// The calling thread's error message (im2win_last_error), shared by the
// translation units that implement entry points.
#pragma once

namespace im2win {

// Sets the message and returns `code`.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Clears the message and returns IM2WIN_OK.
int ok();

}  // namespace im2win
