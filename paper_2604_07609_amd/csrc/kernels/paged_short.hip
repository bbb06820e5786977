// attention over the paged cache, few rows per sequence
#include "../paged_kernels.h"

#define SHORT_KERNEL(HD, BITS, CT, NT)                                                                                                              \
  template <> __global__ void __launch_bounds__(512) __attribute__((amdgpu_num_vgpr(120))) k_paged_short<HD, BITS, CT>(PagedArgs a) { \
    __shared__ ShortShared<HD, CT> sh;                                                                                                                  \
    paged_short<HD, BITS, CT, NT>(a, sh, blockIdx.x, gridDim.x);                                                                                    \
  }
SHORT_KERNEL(64, 16, 1, 4)
SHORT_KERNEL(128, 16, 1, 4)
SHORT_KERNEL(64, 4, 1, 4)
SHORT_KERNEL(128, 4, 1, 4)
SHORT_KERNEL(64, 16, 4, 2)
SHORT_KERNEL(128, 16, 2, 2)
SHORT_KERNEL(64, 4, 4, 4)
SHORT_KERNEL(128, 4, 2, 4)
