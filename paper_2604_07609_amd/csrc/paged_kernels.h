// The kernels of the paged-cache operators, defined in kernels/kv_store.hip, paged_short.hip, paged_prompt.hip and paged_both.hip, and
// those of an engine's phases that are the same operators (kernels/paged_phases.hip).
#pragma once
#include "paged_attention.h"

// Row tiles of the short part beyond one (64 rows with heads of 64, 32 of 128: what the registers hold; 8 sequences of 4000 keys with 32
// rows take 30 us and 60 as prompts, 30 of 2000 in 4 bits with 40 rows 24 and 47), and tiles of keys on their way (two where there are
// more rows: registers; 4 bits with three 122 us, with two 124)
#define SHORT_MORE(HD) ((HD) == 64 ? 4 : 2)
#define SHORT_AHEAD(HD, BITS, CT) ((CT) > 1 ? 2 : (HD) == 128 || (BITS) == 4 ? 3 : 4)
#define PAGED_BOUNDS __launch_bounds__(512) __attribute__((amdgpu_num_vgpr(120)))       // (see PHASE_KERNEL8)
// One row tile over a 4-bit cache is bound by instructions: three workgroups of four waves on a compute unit, else one of eight (128
// sequences of 4096 keys, heads of 128: 122 us and not 131; of 64: 87 and not 100)
#define SHORT_SMALL(BITS, CT) ((BITS) == 4 && (CT) == 1)
#define SHORT_WAVES(BITS, CT) (SHORT_SMALL(BITS, CT) ? 4 : 8)
#define SHORT_PER_CU(BITS, CT) (SHORT_SMALL(BITS, CT) ? 3 : 1)

template <typename T, int HD, int BITS> __global__ void k_kv_store(StoreArgs a);
__global__ void k_kv_read(ReadArgs a, u32 hd);
template <int HD, int BITS, int CT> __global__ void k_paged_short(PagedArgs a);
template <int HD, int BITS> __global__ void k_paged_prompt(PagedArgs a);
template <int HD, int BITS> __global__ void k_paged_both(PagedArgs a);
template <int HD> __global__ void k_paged_merge(PagedArgs a, u32 nwg_prompt);
template <int HD, int BITS> __global__ void k_store_phase(DevCtx c, u32 layer);
template <int HD, int BITS, int CT> __global__ void k_attention_phase(DevCtx c, u32 layer);
