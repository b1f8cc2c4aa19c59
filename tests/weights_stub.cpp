// What the host decides of a call of attention weights (weights_plan.h), for tests without a GPU.  Host code only.
#include "weights_plan.h"

extern "C" int stub_weights_wide(int64_t Tq, int B, int g, int max_rows, int even, int runs) {
  return slh::weights_wide(Tq, B, g, max_rows, even != 0, runs);
}
