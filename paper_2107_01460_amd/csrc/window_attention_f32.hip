// Window attention: the fp32 instances.
#include "window_attention.h"

namespace marl {
void launch_window_f32(const WindowArgs& a, int pass, int waves, unsigned blocks, hipStream_t s) { launch_window<float>(a, pass, waves, blocks, s); }
}  // namespace marl
