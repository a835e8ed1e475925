// Window attention: the bf16 instances.
#include "window_attention.h"

namespace marl {
void launch_window_bf16(const WindowArgs& a, int pass, int waves, unsigned blocks, hipStream_t s) { launch_window<bf16_t>(a, pass, waves, blocks, s); }
}  // namespace marl
