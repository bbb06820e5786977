// attention over the paged cache with groups that share blocks: batches of few rows in all; results joined
#include "../paged_kernels.h"

#define SHARED_SHORT(HD, BITS, CT)                                                                               \
  template <> __global__ void __launch_bounds__(64 * SHORT_WAVES(BITS, CT), SHORT_SMALL(BITS, CT) ? 3 : 2)       \
  __attribute__((amdgpu_num_vgpr(SHORT_SMALL(BITS, CT) ? 84 : 120))) k_shared_short<HD, BITS, CT>(SharedArgs a) {\
    __shared__ ShortShared<HD, CT, SHORT_WAVES(BITS, CT), true> sh;                                              \
    paged_short<HD, BITS, CT, SHORT_AHEAD(HD, BITS, CT), SHORT_WAVES(BITS, CT)>(a, sh, blockIdx.x, gridDim.x);   \
  }
#define SHARED_SHORTS(HD, BITS) SHARED_SHORT(HD, BITS, 1) SHARED_SHORT(HD, BITS, SHORT_MORE(HD))
SHARED_SHORTS(64, 16)
SHARED_SHORTS(128, 16)
SHARED_SHORTS(64, 4)
SHARED_SHORTS(128, 4)

template <int HD>
__device__ __forceinline__ void join_body(const SharedArgs& a, u32 nwg_prompt) {
  __shared__ JoinShared sh;
  shared_join<HD>(a, sh, blockIdx.x, gridDim.x, nwg_prompt);
}
template <> __global__ void __launch_bounds__(512) k_shared_join<64>(SharedArgs a, u32 nwg_prompt) { join_body<64>(a, nwg_prompt); }
template <> __global__ void __launch_bounds__(512) k_shared_join<128>(SharedArgs a, u32 nwg_prompt) { join_body<128>(a, nwg_prompt); }
