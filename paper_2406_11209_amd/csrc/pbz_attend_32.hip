// Attention over a cache of lines of 32: see pbz_attend.h.
#include "pbz_attend.h"

int pbz::launch_attend_32(bool tall, int rows, bool fine, const AttendCall& call, hipStream_t s) {
  return launch<32>(tall, rows, fine, call, s);
}
