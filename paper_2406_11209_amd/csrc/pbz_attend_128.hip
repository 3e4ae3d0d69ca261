// Attention over a cache of lines of 128: see pbz_attend.h.
#include "pbz_attend.h"

int pbz::launch_attend_128(bool tall, int rows, bool fine, const AttendCall& call, hipStream_t s) {
  return launch<128>(tall, rows, fine, call, s);
}
