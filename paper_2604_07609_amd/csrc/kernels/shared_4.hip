// attention over the paged cache with groups that share blocks, in 4 bits
#include "../paged_kernels.h"

#define SHARED_KERNEL(HD, BITS, CT)                                                                    \
  template <> __global__ void PAGED_BOUNDS k_shared_attention<HD, BITS, CT>(SharedArgs a) {            \
    __shared__ SharedKernelRoom<HD, CT> sh;                                                            \
    shared_attention<HD, BITS, CT>(a, sh, blockIdx.x, gridDim.x);                                      \
  }
SHARED_KERNEL(64, 4, ANY_CT)
SHARED_KERNEL(128, 4, ANY_CT)
