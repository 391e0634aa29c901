// The library's one error channel: every entry point reports through it.
#ifndef SDNN_ERROR_H
#define SDNN_ERROR_H

#include "sdnn.h"

namespace sdnn_error {

// Keeps the message that sdnn_last_error() answers on this thread and returns `s`. Throws nothing.
__attribute__((visibility("hidden"), format(printf, 2, 3))) sdnn_status fail(sdnn_status s, const char *fmt, ...);

}  // namespace sdnn_error

#endif  // SDNN_ERROR_H
