// The scan's instances for fp32 elements: products on the fp32 matrix instructions.
#include "linear_attention.h"

namespace marl {
void launch_scan_f32(const ScanArgs& a, int nk, int nv, bool state_only, dim3 grid, dim3 block, hipStream_t s) {
  launch_scan<float>(a, nk, nv, state_only, grid, block, s);
}
}  // namespace marl
