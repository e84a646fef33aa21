// The decode attention's partial phase under score rules: the kernels of
// attention_device.h with RULES, in a file of their own (every cache format is
// compiled twice, and the two halves side by side).
#include "attention_device.h"

namespace mikv {

void launch_partial_rules(const AttnArgs &A, const mikv_cache *c, bool lean, dim3 grid, hipStream_t st) {
  launch_partial_c<true>(A, c, lean, grid, st);
}

}  // namespace mikv
