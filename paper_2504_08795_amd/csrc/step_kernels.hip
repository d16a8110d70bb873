// Kernels of the operators of a generation step but for attention: norm, append and 4-bit products.  Device code only (built as a code
// object that is linked into the library as data); argument blocks are those of step_args.h.
#include "append_kernel.h"
#include "matvec_kernel.h"
#include "norm_kernel.h"

namespace daris {

template <bool BF16, bool F8, bool ALIGNED, int NV, int T>
__global__ __launch_bounds__(T) void step_norm(NormArgs a) { norm_body<BF16, F8, ALIGNED, NV, T>(a); }

template <bool BF16, int D>
__global__ __launch_bounds__(256) void step_append(AppendArgs a) { append_body<BF16, D>(a); }

// ... where rows are nodes of trees
template <bool BF16, int D>
__global__ __launch_bounds__(256) void step_append_tree(TreeAppendArgs a) { append_body<BF16, D, true>(a.append, a.tree); }

template <int XT, int G, bool BF16_OUT>
__global__ __launch_bounds__(kMatvecWaves * 64) void step_matvec(MatvecArgs a) { matvec_body<XT, G, BF16_OUT>(a); }

#define NORM(B, F, A)                                      \
  template __global__ void step_norm<B, F, A, 1, 64>(NormArgs);   \
  template __global__ void step_norm<B, F, A, 1, 256>(NormArgs);  \
  template __global__ void step_norm<B, F, A, 2, 256>(NormArgs);  \
  template __global__ void step_norm<B, F, A, 4, 256>(NormArgs);  \
  template __global__ void step_norm<B, F, A, 4, 1024>(NormArgs); \
  template __global__ void step_norm<B, F, A, 0, 1024>(NormArgs);
NORM(false, false, false) NORM(false, false, true) NORM(false, true, false) NORM(false, true, true)
NORM(true, false, false) NORM(true, false, true) NORM(true, true, false) NORM(true, true, true)

#define APPEND_TREE(B) template __global__ void step_append_tree<B, 64>(TreeAppendArgs); template __global__ void step_append_tree<B, 128>(TreeAppendArgs); template __global__ void step_append_tree<B, 256>(TreeAppendArgs);
APPEND_TREE(false) APPEND_TREE(true)

#define APPEND(B) template __global__ void step_append<B, 64>(AppendArgs); template __global__ void step_append<B, 128>(AppendArgs); template __global__ void step_append<B, 256>(AppendArgs);
APPEND(false) APPEND(true)

#define MATVEC(X, O) template __global__ void step_matvec<X, 32, O>(MatvecArgs); template __global__ void step_matvec<X, 64, O>(MatvecArgs); template __global__ void step_matvec<X, 128, O>(MatvecArgs);
MATVEC(kRowsF32, false) MATVEC(kRowsBf16, true) MATVEC(kRowsF8, false) MATVEC(kRowsF8, true)

}  // namespace daris
