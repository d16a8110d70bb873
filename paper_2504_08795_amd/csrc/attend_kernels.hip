// Kernels of attention over the paged cache (device code only, built as a code object that is linked into the library as data).
#include <type_traits>

#include "attend_kernel.h"

namespace daris {

template <bool BF16, int D>
__global__ __launch_bounds__(256) void step_attend_narrow(AttendArgs a) { attend_narrow_body<BF16, D>(a); }
template <bool BF16, int D>
__global__ __launch_bounds__(256, BF16 ? 2 : 1) void step_attend_wide(AttendArgs a) { attend_wide_body<BF16, D>(a); }

// ... where the step's rows are nodes of trees
template <bool BF16, int D>
__global__ __launch_bounds__(256, BF16 && D < 256 ? 2 : 1) void step_attend_tree_narrow(TreeAttendArgs a) { attend_narrow_body<BF16, D, true>(a.attend, a.tree); }
template <bool BF16, int D>
__global__ __launch_bounds__(256, BF16 ? 2 : 1) void step_attend_tree_wide(TreeAttendArgs a) { attend_wide_body<BF16, D, true>(a.attend, a.tree); }

#define NARROW(B, D) template __global__ void step_attend_narrow<B, D>(AttendArgs); template __global__ void step_attend_tree_narrow<B, D>(TreeAttendArgs);
#define WIDE(B, D) template __global__ void step_attend_wide<B, D>(AttendArgs);
#define TREE_WIDE(B, D) template __global__ void step_attend_tree_wide<B, D>(TreeAttendArgs);
NARROW(false, 64) NARROW(false, 128) NARROW(false, 256) NARROW(true, 64) NARROW(true, 128) NARROW(true, 256)
// (queries of 256 channels do not fit a wave's registers beside 32 columns of outputs)
WIDE(false, 64) WIDE(false, 128) WIDE(true, 64) WIDE(true, 128)
// (fp32's of 128 have a CU for themselves, and a tree's columns seldom fill them: 32 trees of up to 64 nodes behind up to 4096 tokens, 32 query and 8 key heads, 148 us a call
// narrow and 232 wide; 32 of 128 behind 2500, 200 and 212)
TREE_WIDE(false, 64) TREE_WIDE(true, 64) TREE_WIDE(true, 128)

}  // namespace daris
