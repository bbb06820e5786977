// attention over the paged cache, few rows per sequence
#include "../paged_kernels.h"

#define SHORT_KERNEL(HD, BITS, CT)                                                                     \
  template <> __global__ void PAGED_BOUNDS k_paged_short<HD, BITS, CT>(PagedArgs a) {                  \
    __shared__ ShortShared<HD, CT> sh;                                                                 \
    paged_short<HD, BITS, CT, SHORT_AHEAD(HD, BITS, CT)>(a, sh, blockIdx.x, gridDim.x);                \
  }
#define SHORT_KERNELS(HD, BITS) SHORT_KERNEL(HD, BITS, 1) SHORT_KERNEL(HD, BITS, SHORT_MORE(HD))
SHORT_KERNELS(64, 16)
SHORT_KERNELS(128, 16)
SHORT_KERNELS(64, 4)
SHORT_KERNELS(128, 4)
