// attention over the paged cache with groups that share blocks, in halves
#include "../paged_kernels.h"

#define SHARED_KERNEL(HD, BITS, CT)                                                                    \
  template <> __global__ void PAGED_BOUNDS k_shared_attention<HD, BITS, CT>(SharedArgs a) {            \
    __shared__ SharedKernelRoom<HD, CT> sh;                                                            \
    shared_attention<HD, BITS, CT>(a, sh, blockIdx.x, gridDim.x);                                      \
  }
SHARED_KERNEL(64, 16, ANY_CT)
SHARED_KERNEL(128, 16, 1)
SHARED_KERNEL(128, 16, SHORT_MORE(128))

template <int HD>
__device__ __forceinline__ void join_body(const SharedArgs& a) { shared_join<HD>(a, blockIdx.x * (BLK_THREADS / 64) + (threadIdx.x >> 6)); }
template <> __global__ void __launch_bounds__(BLK_THREADS) k_shared_join<64>(SharedArgs a) { join_body<64>(a); }
template <> __global__ void __launch_bounds__(BLK_THREADS) k_shared_join<128>(SharedArgs a) { join_body<128>(a); }
