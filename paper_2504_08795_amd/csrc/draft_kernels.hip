// Kernels of the operators behind a drafted step: sampling, acceptance, and tokens and pages that change their place in the cache (device code
// only, built as a code object that is linked into the library as data).
#include "accept_kernel.h"
#include "move_kernel.h"
#include "sample_kernel.h"

namespace daris {

template <bool BF16>
__global__ __launch_bounds__(kSampleThreads) void step_sample(SampleArgs a) { sample_body<BF16, true>(a); }
template <bool BF16>
__global__ __launch_bounds__(kSampleThreads, BF16 ? 8 : 4) void step_sample_parts(SampleArgs a) { sample_body<BF16, false>(a); }
__global__ __launch_bounds__(64) void step_accept(AcceptArgs a) { accept_body(a); }
template <int D>
__global__ __launch_bounds__(256) void step_keep(KeepArgs a) { keep_body<D>(a); }
template <int D>
__global__ __launch_bounds__(256) void step_copy(CopyArgs a) { copy_body<D>(a); }

template __global__ void step_sample<false>(SampleArgs);
template __global__ void step_sample<true>(SampleArgs);
template __global__ void step_sample_parts<false>(SampleArgs);
template __global__ void step_sample_parts<true>(SampleArgs);
template __global__ void step_keep<64>(KeepArgs);
template __global__ void step_keep<128>(KeepArgs);
template __global__ void step_keep<256>(KeepArgs);
template __global__ void step_copy<64>(CopyArgs);
template __global__ void step_copy<128>(CopyArgs);
template __global__ void step_copy<256>(CopyArgs);

}  // namespace daris
