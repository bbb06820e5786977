// attention over the paged cache, batches of single tokens and prompts
#include "../paged_kernels.h"

#define BOTH_KERNEL(HD, BITS)                                                                          \
  template <> __global__ void PAGED_BOUNDS k_paged_both<HD, BITS>(PagedArgs a) {                       \
    __shared__ PagedShared<HD, 1> sh;                                                                  \
    paged_both<HD, BITS, 1, SHORT_AHEAD(HD, BITS, 1)>(a, sh, blockIdx.x, gridDim.x);                   \
  }
BOTH_KERNEL(64, 16)
BOTH_KERNEL(128, 16)
BOTH_KERNEL(64, 4)
BOTH_KERNEL(128, 4)
