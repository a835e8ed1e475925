// The scan's instances for fp32 elements: products on the fp32 matrix instructions.
#include "linear_attention.h"

namespace marl {
void launch_scan_f32(const ScanArgs& a, int dx, int dz, bool state_only, hipStream_t s) { launch_scan<float>(a, dx, dz, state_only, s); }
}  // namespace marl
