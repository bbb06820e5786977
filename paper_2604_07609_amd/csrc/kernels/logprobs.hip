// log probabilities, ranks, entropy and most probable tokens
#include "../paged_kernels.h"

#define LOGPROBS_KERNEL(T, TOP)                                                                                   \
  template <> __global__ void __launch_bounds__(BLK_THREADS, 4) k_token_logprobs<T, TOP>(LogprobArgs a) {         \
    __shared__ LogprobShared<TOP> sh;                                                                                \
    token_logprobs<T, TOP>(a, sh, blockIdx.x);                                                                    \
  }
#define LOGPROBS_KERNELS(T) LOGPROBS_KERNEL(T, false) LOGPROBS_KERNEL(T, true)
LOGPROBS_KERNELS(float)
LOGPROBS_KERNELS(_Float16)
LOGPROBS_KERNELS(__bf16)
