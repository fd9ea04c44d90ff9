// fa_generic.hip -- attention forward with fp32 weights (fa_generic_kernel.h) over
// all keys, causal or not.
#include "fa_generic_kernel.h"

namespace fa {

hipError_t launch_generic(const Problem &p, hipStream_t stream) { return launch_types<false>(p, stream); }

}  // namespace fa
