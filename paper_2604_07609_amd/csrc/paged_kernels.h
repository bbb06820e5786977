// The kernels of the paged-cache operators, defined in kernels/kv_store.hip, paged_short.hip and paged_prompt.hip.
#pragma once
#include "paged_attention.h"

#define STORE_UNROLL 2                                 // rows of a lane group on their way at a time
template <typename T, int HD, int BITS> __global__ void k_kv_store(StoreArgs a);
__global__ void k_kv_read(ReadArgs a, u32 hd);
template <int HD, int BITS, int CT> __global__ void k_paged_short(PagedArgs a);
template <int HD, int BITS> __global__ void k_paged_prompt(PagedArgs a);
template <int HD> __global__ void k_paged_merge(PagedArgs a, u32 nwg_prompt);
