// A stand-in for the HIP runtime and the attention kernels: says what the entry points of attend_api.cpp
// would launch for a card of 256 compute units.  Host code only.
#include <cstdio>
#include <string>

#include "attend.h"

static std::string g_log;

static void note(const char* what, const slh::AttendArgs& a, bool paged, int rows, long blocks) {
  char line[200];
  snprintf(line, sizeof line, "%s %d %d %ld %d %d %d %d\n", what, (int)paged, rows, blocks, a.splits, a.pre_tiles, a.pre_splits, a.chain);
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
hipError_t launch_attend_tiles(const AttendArgs& a, bool paged, bool, int rows, int, int64_t blocks, hipStream_t) {
  note("tiles", a, paged, rows, blocks);
  return hipSuccess;
}
hipError_t launch_attend_rows(const AttendArgs& a, bool paged, bool, int rows, int, int64_t blocks, hipStream_t) {
  note("rows", a, paged, rows, blocks);
  return hipSuccess;
}
hipError_t launch_attend_both(const AttendArgs& a, bool, int rows, int, int64_t, int64_t blocks, hipStream_t) {
  note("both", a, true, rows, blocks);
  return hipSuccess;
}
hipError_t launch_attend_join(const AttendArgs& a, bool, int, int slots, hipStream_t) {
  note("join", a, false, slots, a.rows);
  return hipSuccess;
}
}  // namespace slh
