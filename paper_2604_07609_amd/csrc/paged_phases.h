// The paged-cache operators as phases of an engine's iteration (models with per-head norms, a window or a 4-bit cache): shapes come from
// the device metadata that the scheduler step has written.
#pragma once
#include "paged_kernels.h"
#include "phases.h"

template <int HD, int BITS>
__device__ __forceinline__ void store_phase(const DevCtx& c, u32 layer, ValueShared<HD>& sh, u32 wg, u32 nwg) {
  const IterMeta* m = c.meta;
  if (m->skip || m->kind == KIND_IDLE) return;
  const LayerW* L = c.layers + layer;
  StoreArgs a{};
  a.q = c.qkv; a.k = c.qkv + c.nq * HD; a.v = c.qkv + (c.nq + c.nkv) * HD;
  a.qs = a.ks = a.vs = c.qkv_n;
  a.qg = L->gq; a.kg = L->gk; a.pos = c.positions; a.slot = c.slot_mapping; a.tab = c.rope_tab; a.rows = c.max_seq_len;
  a.qo = c.qbuf; a.qos = (u64)c.nq * HD; a.cache = (char*)c.kv + layer * c.kv_layer_bytes; a.n_blocks = c.n_blocks; a.nq = c.nq; a.nkv = c.nkv; a.T = m->n_tokens;
  a.eps = c.eps; a.q_scale = 1.0f / sqrtf((float)HD); a.group = store_group(a.T, c.nkv, c.n_cu);
  const u32 total = store_wgs(a.T, a.nq, a.nkv, HD, BITS, a.group);
  for (u32 x = wg; x < total; x += nwg) kv_store<float, HD, BITS>(a, sh, x);      // (a wave's part of the LDS is its own)
}
template <int HD, int BITS, int CT>
__device__ __forceinline__ void attention_phase(const DevCtx& c, u32 layer, PagedShared<HD, CT>& sh, u32 wg, u32 nwg) {
  const IterMeta* m = c.meta;
  if (m->skip || m->kind == KIND_IDLE) return;
  PagedArgs a{};
  a.q = c.qbuf; a.qs = (u64)c.nq * HD; a.out = c.aq; a.out_tbs = c.TBS; a.cu = (const i32*)c.cu_seqlens; a.lens = (const i32*)c.seq_len;
  a.tables = c.block_tables; a.table_row = c.seq_bslot; a.cache = (const char*)c.kv + layer * c.kv_layer_bytes; a.n_blocks = c.n_blocks; a.max_blocks = c.max_blocks_per_seq;
  a.nq = c.nq; a.nkv = c.nkv; a.G = c.nq / c.nkv; a.n_seqs = m->n_seqs; a.n_tokens = m->n_tokens; a.max_q = m->n_tokens;
  a.window = c.window; a.sinks = c.sinks; a.c = 1.44269504088896340736f; a.short_rows = 16 * CT; a.n_splits = 1;
  a.ctr = c.paged_ctr; a.part = c.paged_part;
  paged_both<HD, BITS, CT, SHORT_AHEAD(HD, BITS, CT)>(a, sh, wg, nwg);
}

#define ATTENTION_PHASE(HD, BITS, CT)                                                                                     \
  template <> __global__ void PAGED_BOUNDS k_attention_phase<HD, BITS, CT>(DevCtx c, u32 layer) {                         \
    __shared__ PagedShared<HD, CT> sh;                                                                                    \
    attention_phase<HD, BITS, CT>(c, layer, sh, blockIdx.x, gridDim.x);                                                   \
  }
#define PAGED_PHASES(HD, BITS)                                                                                            \
  template <> __global__ void __launch_bounds__(BLK_THREADS, 2) k_store_phase<HD, BITS>(DevCtx c, u32 layer) {            \
    __shared__ ValueShared<HD> sh;                                                                                        \
    store_phase<HD, BITS>(c, layer, sh, blockIdx.x, gridDim.x);                                                           \
  }                                                                                                                       \
  ATTENTION_PHASE(HD, BITS, 1) ATTENTION_PHASE(HD, BITS, SHORT_MORE(HD))
