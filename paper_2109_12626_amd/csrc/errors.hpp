// The calling thread's last error (dpar_last_error), for every source file of
// entry points.
#pragma once

namespace dpar {

// Keeps the text and returns the code.
int set_error(int code, const char* text);

}  // namespace dpar
