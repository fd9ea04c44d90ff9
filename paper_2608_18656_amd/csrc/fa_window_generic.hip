// fa_window_generic.hip -- attention with a sliding window and first keys that
// stay visible, with fp32 weights (fa_generic_kernel.h): fp32 inputs, head sizes
// other than 64 and 128, key rows too long for the half-precision kernels.
#include "fa_generic_kernel.h"

namespace fa {

hipError_t launch_generic_window(const Problem &p, hipStream_t stream) { return launch_types<true>(p, stream); }

}  // namespace fa
