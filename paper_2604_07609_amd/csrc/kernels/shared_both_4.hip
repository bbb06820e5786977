// attention over the paged cache with groups that share blocks, in 4 bits: few rows and many
#include "../paged_kernels.h"

#define SHARED_BOTH(HD, BITS, CT)                                                                      \
  template <> __global__ void PAGED_BOUNDS k_shared_both<HD, BITS, CT>(SharedArgs a) {                 \
    __shared__ PagedShared<HD, CT, SharedArgs> sh;                                                     \
    paged_both<HD, BITS, CT, SHORT_AHEAD(HD, BITS, CT)>(a, sh, blockIdx.x, gridDim.x);                 \
  }
SHARED_BOTH(64, 4, 1)
SHARED_BOTH(64, 4, SHORT_MORE(64))
SHARED_BOTH(128, 4, 1)
SHARED_BOTH(128, 4, SHORT_MORE(128))
