// Kernels of attention over the paged cache (device code only, built as a code object that is linked into the library as data).
#include <type_traits>

#include "attend_kernel.h"

namespace daris {

template <bool BF16, int D>
__global__ __launch_bounds__(256) void step_attend_narrow(AttendArgs a) { attend_narrow_body<BF16, D>(a); }
template <bool BF16, int D>
__global__ __launch_bounds__(256, BF16 ? 2 : 1) void step_attend_wide(AttendArgs a) { attend_wide_body<BF16, D>(a); }

#define NARROW(B, D) template __global__ void step_attend_narrow<B, D>(AttendArgs);
#define WIDE(B, D) template __global__ void step_attend_wide<B, D>(AttendArgs);
NARROW(false, 64) NARROW(false, 128) NARROW(false, 256) NARROW(true, 64) NARROW(true, 128) NARROW(true, 256)
// (queries of 256 channels do not fit a wave's registers beside 32 columns of outputs)
WIDE(false, 64) WIDE(false, 128) WIDE(true, 64) WIDE(true, 128)

}  // namespace daris
