// attention over the paged cache, few rows per sequence
#include "../paged_kernels.h"

#define SHORT_KERNEL(HD, BITS, CT)                                                                              \
  template <> __global__ void __launch_bounds__(64 * SHORT_WAVES(BITS, CT), SHORT_SMALL(BITS, CT) ? 3 : 2)      \
  __attribute__((amdgpu_num_vgpr(SHORT_SMALL(BITS, CT) ? 84 : 120))) k_paged_short<HD, BITS, CT>(PagedArgs a) { \
    __shared__ ShortShared<HD, CT, SHORT_WAVES(BITS, CT)> sh;                                                   \
    paged_short<HD, BITS, CT, SHORT_AHEAD(HD, BITS, CT), SHORT_WAVES(BITS, CT)>(a, sh, blockIdx.x, gridDim.x);  \
  }
#define SHORT_KERNELS(HD, BITS) SHORT_KERNEL(HD, BITS, 1) SHORT_KERNEL(HD, BITS, SHORT_MORE(HD))
SHORT_KERNELS(64, 16)
SHORT_KERNELS(128, 16)
SHORT_KERNELS(64, 4)
SHORT_KERNELS(128, 4)
