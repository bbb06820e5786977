// attention over the paged cache, many rows per sequence
#include "../paged_kernels.h"

#define PROMPT_KERNEL(HD, BITS)                                                                        \
  template <> __global__ void PAGED_BOUNDS k_paged_prompt<HD, BITS>(PagedArgs a) {                     \
    __shared__ PromptShared sh;                                                                        \
    paged_prompt<HD, BITS>(a, sh, blockIdx.x, gridDim.x, false);                                       \
  }
PROMPT_KERNEL(64, 16)
PROMPT_KERNEL(128, 16)
PROMPT_KERNEL(64, 4)
PROMPT_KERNEL(128, 4)

template <int HD>
__device__ __forceinline__ void merge_body(const PagedArgs& a, u32 nwg_prompt) {
  __shared__ PromptMergeShared sh;
  prompt_merge<HD>(a, sh, blockIdx.x, gridDim.x, nwg_prompt);
}
template <> __global__ void __launch_bounds__(512) k_paged_merge<64>(PagedArgs a, u32 nwg_prompt) { merge_body<64>(a, nwg_prompt); }
template <> __global__ void __launch_bounds__(512) k_paged_merge<128>(PagedArgs a, u32 nwg_prompt) { merge_body<128>(a, nwg_prompt); }
