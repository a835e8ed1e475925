// The scan's instances for bf16 elements.
#include "linear_attention.h"

namespace marl {
void launch_scan_bf16(const ScanArgs& a, int nk, int nv, bool state_only, dim3 grid, dim3 block, hipStream_t s) {
  launch_scan<bf16_t>(a, nk, nv, state_only, grid, block, s);
}
}  // namespace marl
