// A stand-in for the HIP runtime and the kernels of 8-bit attention: says what the entry points of attend8_api.cpp
// would launch for a card of 256 compute units.  Host code only.
#include <cstdio>
#include <string>

#include "attend8.h"

static std::string g_log;

static void note(const char* what, const slh::AttendArgs& a, int rows, long blocks) {
  char line[200];
  snprintf(line, sizeof line, "%s %d %ld %d %d %d %d\n", what, rows, blocks, a.splits, a.pre_tiles, a.pre_splits, a.chain);
  g_log += line;
}

extern "C" {
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* n, hipDeviceAttribute_t, int) { *n = 256; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* stub_log() { return g_log.c_str(); }
void stub_clear() { g_log.clear(); }
}

namespace slh {
hipError_t launch_tiles8(const Attend8Args& a, bool, int, int64_t blocks, hipStream_t) {
  note("tiles", a.a, AT_ROWS, blocks);
  return hipSuccess;
}
hipError_t launch_rows8(const Attend8Args& a, bool, int rows, int, int64_t blocks, hipStream_t) {
  note("rows", a.a, rows, blocks);
  return hipSuccess;
}
hipError_t launch_both8(const Attend8Args& a, bool, int rows, int, int64_t, int64_t blocks, hipStream_t) {
  note("both", a.a, rows, blocks);
  return hipSuccess;
}
hipError_t launch_attend_join(const AttendArgs& a, bool, int, int slots, hipStream_t) {
  note("join", a, slots, a.rows);
  return hipSuccess;
}
}  // namespace slh
