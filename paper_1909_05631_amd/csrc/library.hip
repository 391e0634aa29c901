// The network's source as it is, and the door through which the other sources of the library reach its message for
// sdnn_last_error(), which is private to it.
#include "sdnn.hip"

#include "error.h"

sdnn_status sdnn_error::fail(sdnn_status s, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return ::fail(s, "%s", buf);
}
