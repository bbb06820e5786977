// norms, rotation and storage of queries, keys and values; tokens read back
#include "../paged_kernels.h"

#define STORE_KERNEL(T, HD, BITS)                                                                                 \
  template <> __global__ void __launch_bounds__(BLK_THREADS) k_kv_store<T, HD, BITS>(StoreArgs a) {               \
    __shared__ ValueShared<HD> sh;                                                                                \
    kv_store<T, HD, BITS>(a, sh, blockIdx.x);                                                       \
  }
#define STORE_KERNELS(T) STORE_KERNEL(T, 64, 16) STORE_KERNEL(T, 128, 16) STORE_KERNEL(T, 64, 4) STORE_KERNEL(T, 128, 4)
STORE_KERNELS(float)
STORE_KERNELS(_Float16)
STORE_KERNELS(__bf16)

__global__ void __launch_bounds__(BLK_THREADS) k_kv_read(ReadArgs a, u32 hd) {
  const u64 i = (u64)blockIdx.x * BLK_THREADS + threadIdx.x;
  if (hd == 64) kv_read<64>(a, i); else kv_read<128>(a, i);
}
