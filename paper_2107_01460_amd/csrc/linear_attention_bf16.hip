// The scan's instances for bf16 elements.
#include "linear_attention.h"

namespace marl {
void launch_scan_bf16(const ScanArgs& a, int dx, int dz, bool state_only, hipStream_t s) { launch_scan<bf16_t>(a, dx, dz, state_only, s); }
}  // namespace marl
