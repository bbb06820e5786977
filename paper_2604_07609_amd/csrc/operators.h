// Host side of the device-memory operators of the C ABI: argument checks, launch shapes, workspaces. Included by blink.hip.
#pragma once
#include "paged_kernels.h"

// The calling thread's device for the length of a call.
struct OnDevice {
  int before = -1;
  hipError_t err = hipSuccess;
  explicit OnDevice(int device) {
    int now = -1;
    err = hipGetDevice(&now);
    if (err == hipSuccess && now != device) { err = hipSetDevice(device); before = now; }
  }
  ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};
static int compute_units(int device, u32* n) {       // asked once per device
  static std::atomic<int> known[64];
  int v = device >= 0 && device < 64 ? known[device].load(std::memory_order_relaxed) : 0;
  if (!v) {
    int n_dev = 0;
    if (hipGetDeviceCount(&n_dev) != hipSuccess || n_dev <= 0) return fail(BLINK_ERR_DEVICE, "no HIP device available");
    if (device < 0 || device >= n_dev) return fail(BLINK_ERR_INVAL, "device %d out of range", device);
    HIPCHK(hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, device));
    if (device < 64) known[device].store(v, std::memory_order_relaxed);
  }
  *n = (u32)v;
  return BLINK_OK;
}

static int check_cache(const blink_kv_cache& c) {
  if (c.bits != 16 && c.bits != 4) return fail(BLINK_ERR_INVAL, "a cache holds 16 or 4 bits, not %u", c.bits);
  if (c.head_dim != 64 && c.head_dim != 128) return fail(BLINK_ERR_INVAL, "head_dim must be 64 or 128");
  if (!c.n_blocks || !c.n_kv_heads || c.n_kv_heads > 1024) return fail(BLINK_ERR_INVAL, "n_blocks must be positive and n_kv_heads in [1, 1024]");
  if (c.n_blocks > (1u << 27)) return fail(BLINK_ERR_TOO_LARGE, "more than 2^27 blocks: places do not fit 32 bits");
  return BLINK_OK;
}
static int check_heads(const blink_kv_cache& c, u32 nq) {
  if (int rc = check_cache(c)) return rc;
  if (!c.data || (u64)c.data % 256) return fail(BLINK_ERR_INVAL, "the cache's data must be aligned to 256 bytes");
  if (!nq || nq % c.n_kv_heads || nq / c.n_kv_heads > 64) return fail(BLINK_ERR_INVAL, "n_q_heads must be a multiple (at most 64) of n_kv_heads");
  return BLINK_OK;
}
// a matrix of rows that kernels read or write 16 bytes at a time
static int check_rows(const char* name, const void* p, u64 stride, u64 width, u32 elem) {
  if (!p) return fail(BLINK_ERR_INVAL, "%s is null", name);
  if ((u64)p % 16 || stride * elem % 16) return fail(BLINK_ERR_INVAL, "%s: rows must be aligned to 16 bytes", name);
  if (stride < width) return fail(BLINK_ERR_INVAL, "%s: a stride of %llu elements, rows are %llu long", name, (unsigned long long)stride, (unsigned long long)width);
  return BLINK_OK;
}

constexpr u32 LAUNCH_WGS = 0xFFFFFFFFu / BLK_THREADS;     // workgroups of a launch, whose threads are counted in 32 bits

extern "C" int blink_kv_cache_bytes(uint32_t n_blocks, uint32_t n_kv_heads, uint32_t head_dim, uint32_t bits, uint64_t* bytes) {
  g_err.clear();
  if (!bytes) return fail(BLINK_ERR_INVAL, "null argument");
  const blink_kv_cache c{nullptr, n_blocks, n_kv_heads, head_dim, bits};
  if (int rc = check_cache(c)) return rc;
  *bytes = (u64)n_blocks * n_kv_heads * (bits == 16 ? 64 : 17) * head_dim;
  return BLINK_OK;
}

template <typename T>
static hipError_t launch_store(const StoreArgs& s, u32 hd, u32 bits, u32 grid, hipStream_t st) {
  if (hd == 64) return bits == 16 ? launch(k_kv_store<T, 64, 16>, grid, BLK_THREADS, st, s) : launch(k_kv_store<T, 64, 4>, grid, BLK_THREADS, st, s);
  return bits == 16 ? launch(k_kv_store<T, 128, 16>, grid, BLK_THREADS, st, s) : launch(k_kv_store<T, 128, 4>, grid, BLK_THREADS, st, s);
}
extern "C" int blink_qk_norm_rope(int32_t device, const blink_qk_norm_rope_args* a, void* stream) {
  g_err.clear();
  if (!a) return fail(BLINK_ERR_INVAL, "null argument");
  if (int rc = check_heads(a->cache, a->n_q_heads)) return rc;
  if (a->in_type > BLINK_TYPE_BF16) return fail(BLINK_ERR_INVAL, "in_type must be BLINK_TYPE_FLOAT, BLINK_TYPE_HALF or BLINK_TYPE_BF16");
  const u32 hd = a->cache.head_dim, nkv = a->cache.n_kv_heads, es = a->in_type == BLINK_TYPE_FLOAT ? 4 : 2;
  if (!(a->eps >= 0.f)) return fail(BLINK_ERR_INVAL, "eps must not be negative");
  if (a->n_tokens == 0) return BLINK_OK;
  if ((u64)a->n_tokens * (a->n_q_heads + 2ull * nkv) >= (1ull << 31)) return fail(BLINK_ERR_TOO_LARGE, "2^31 rows or more");
  // (so many tokens have the largest groups, whatever the number of compute units)
  if (store_wgs(a->n_tokens, a->n_q_heads, nkv, hd, a->cache.bits, STORE_GROUP) > LAUNCH_WGS) return fail(BLINK_ERR_TOO_LARGE, "too many tokens for one call");
  if (int rc = check_rows("q", a->q, a->q_stride, (u64)a->n_q_heads * hd, es)) return rc;
  if (int rc = check_rows("k", a->k, a->k_stride, (u64)nkv * hd, es)) return rc;
  if (int rc = check_rows("v", a->v, a->v_stride, (u64)nkv * hd, es)) return rc;
  if (int rc = check_rows("q_out", a->q_out, a->q_out_stride, (u64)a->n_q_heads * hd, 2)) return rc;
  if (!a->positions || !a->slots || !a->rope_table) return fail(BLINK_ERR_INVAL, "positions, slots and rope_table must not be null");
  if ((u64)a->rope_table % 16 || (u64)a->q_gain % 16 || (u64)a->k_gain % 16 || (u64)a->positions % 4 || (u64)a->slots % 4)
    return fail(BLINK_ERR_INVAL, "rope_table and gains must be aligned to 16 bytes, positions and slots to 4");
  if (!a->rope_rows) return fail(BLINK_ERR_INVAL, "rope_rows must be positive");
  u32 n_cu;
  if (int rc = compute_units(device, &n_cu)) return rc;
  OnDevice on(device);
  HIPCHK(on.err);
  StoreArgs s{};
  s.q = a->q; s.k = a->k; s.v = a->v; s.qs = a->q_stride; s.ks = a->k_stride; s.vs = a->v_stride;
  s.qg = a->q_gain; s.kg = a->k_gain; s.pos = a->positions; s.slot = a->slots; s.tab = (const float2*)a->rope_table; s.rows = a->rope_rows;
  s.qo = (f16_t*)a->q_out; s.qos = a->q_out_stride; s.cache = a->cache.data; s.n_blocks = a->cache.n_blocks; s.nq = a->n_q_heads; s.nkv = nkv; s.T = a->n_tokens;
  s.eps = a->eps; s.q_scale = a->q_scale; s.group = store_group(s.T, nkv, n_cu);
  const u32 grid = store_wgs(s.T, s.nq, nkv, hd, a->cache.bits, s.group);
  const hipStream_t st = (hipStream_t)stream;
  HIPCHK(a->in_type == BLINK_TYPE_FLOAT ? launch_store<float>(s, hd, a->cache.bits, grid, st)
         : a->in_type == BLINK_TYPE_HALF ? launch_store<_Float16>(s, hd, a->cache.bits, grid, st) : launch_store<__bf16>(s, hd, a->cache.bits, grid, st));
  return BLINK_OK;
}

extern "C" int blink_kv_cache_read(int32_t device, const blink_kv_cache* c, const int32_t* slots, uint32_t n_tokens, void* k_out, void* v_out, void* stream) {
  g_err.clear();
  if (!c) return fail(BLINK_ERR_INVAL, "null argument");
  if (int rc = check_heads(*c, c->n_kv_heads)) return rc;
  if (n_tokens == 0) return BLINK_OK;
  const u64 width = (u64)c->n_kv_heads * c->head_dim, n = n_tokens * width / 8;
  if (int rc = check_rows("k_out", k_out, width, width, 2)) return rc;
  if (int rc = check_rows("v_out", v_out, width, width, 2)) return rc;
  if (!slots || (u64)slots % 4) return fail(BLINK_ERR_INVAL, "slots is null or not aligned");
  if (n > (u64)LAUNCH_WGS * BLK_THREADS) return fail(BLINK_ERR_TOO_LARGE, "too many tokens for one call");
  u32 n_cu;
  if (int rc = compute_units(device, &n_cu)) return rc;
  OnDevice on(device);
  HIPCHK(on.err);
  const ReadArgs r{c->data, c->bits, c->n_blocks, c->n_kv_heads, n_tokens, slots, (f16_t*)k_out, (f16_t*)v_out};
  HIPCHK(launch(k_kv_read, (u32)((n + BLK_THREADS - 1) / BLK_THREADS), BLK_THREADS, (hipStream_t)stream, r, c->head_dim));
  return BLINK_OK;
}

// ---- attention ------------------------------------------------------------------------------------------------------------------
// The workspace: the counters, then results of the short part, then those of the prompt part. The counters are zeros between calls and results
// are anything, so where the ones end must be the same in every call, whatever its batch, heads, bits and plan: the counters of
// the launch with the most workgroups, in whole 8 KiB.
static u64 paged_ctr_bytes(u32 n_cu) { return (paged_counters(n_cu * SHORT_PER_CU(4, 1)) * 4ull + 8191) / 8192 * 8192; }
// Which kernels a call takes, from what the host knows: its longest run of queries, and not which sequences have it.
struct PagedPlan {
  u32 ct;                 // row tiles of the short part (0: there is none)
  u32 short_rows;         // sequences with at most so many rows are its
  bool prompt;            // there is a prompt part (with a short one: in one launch)
  u32 wgs, threads, n_splits;
  u64 part_bytes, prompt_bytes;
  u64 bytes(u32 n_cu) const { return paged_ctr_bytes(n_cu) + part_bytes + prompt_bytes; }
};
static PagedPlan paged_plan(u32 hd, u32 bits, u32 nq, u32 nkv, u32 n_seqs, u32 n_tokens, u32 max_q, u32 key_steps, u32 n_cu) {
  PagedPlan p{};
  const u32 G = nq / nkv, most = 16u * SHORT_MORE(hd);       // rows that the short part's registers hold
  const u64 rows = (u64)max_q * G;
  if (rows <= most) { p.ct = rows <= 16 ? 1 : most / 16; p.short_rows = 16 * p.ct; }
  else {
    // (one sequence, or all of one length: the prompt part takes a shorter one just as well, and a launch is saved)
    p.prompt = true;
    if (G <= 16 && n_tokens < (u64)n_seqs * max_q) { p.ct = 1; p.short_rows = 16; }
  }
  p.wgs = n_cu * (p.prompt ? 1 : SHORT_PER_CU(bits, p.ct));
  p.threads = 64 * (p.prompt ? PAGED_WAVES : SHORT_WAVES(bits, p.ct));
  // parts of 256 keys at least, where the items are too few for the chip (64 queries at 8192 keys: 45 us, of 1024 at least 49, in one
  // part 212; parts of 128 gain nothing and need twice the adding up)
  const bool few = (u64)n_tokens * G / PROMPT_ROWS * nkv < p.wgs;
  p.n_splits = p.prompt && few ? std::max(1u, key_steps / 4) : 1u;
  p.part_bytes = p.ct ? short_floats(p.wgs, hd, p.ct) * 4 : 0;
  p.prompt_bytes = p.prompt ? (u64)p.wgs * PROMPT_SLOT(hd) * 4 : 0;
  return p;
}
static int paged_check(const blink_kv_cache& c, u32 nq, u32 n_seqs, u32 max_q) {
  if (!nq || nq % c.n_kv_heads || nq / c.n_kv_heads > 64) return fail(BLINK_ERR_INVAL, "n_q_heads must be a multiple (at most 64) of n_kv_heads");
  if (n_seqs > PAGED_MAX_SEQS) return fail(BLINK_ERR_TOO_LARGE, "%u sequences, at most %u in one call", n_seqs, PAGED_MAX_SEQS);
  if (!max_q || max_q >= (1u << 24)) return fail(BLINK_ERR_INVAL, "max_q must be in [1, 2^24)");
  return BLINK_OK;
}

extern "C" int blink_attention_workspace_bytes(int32_t device, const blink_kv_cache* c, uint32_t n_q_heads, uint32_t n_seqs, uint32_t max_q, uint64_t* bytes) {
  g_err.clear();
  if (!c || !bytes) return fail(BLINK_ERR_INVAL, "null argument");
  if (int rc = check_cache(*c)) return rc;
  if (int rc = paged_check(*c, n_q_heads, n_seqs, max_q)) return rc;
  u32 n_cu;
  if (int rc = compute_units(device, &n_cu)) return rc;
  // (n_tokens below n_seqs * max_q: the larger of the two kinds of launches; and what a smaller max_q would need)
  const PagedPlan p = paged_plan(c->head_dim, c->bits, n_q_heads, c->n_kv_heads, n_seqs, 0, max_q, 1, n_cu);
  const u32 one = n_cu * SHORT_PER_CU(c->bits, 1), more = SHORT_MORE(c->head_dim);
  const u64 least = std::max(short_floats(one, c->head_dim, 1), short_floats(n_cu, c->head_dim, more)) * 4;
  *bytes = std::max(p.bytes(n_cu), paged_ctr_bytes(n_cu) + least);
  return BLINK_OK;
}

template <int HD, int BITS>
static hipError_t launch_paged(const PagedArgs& args, const PagedPlan& plan, hipStream_t st) {
  if (!plan.prompt) return plan.ct == 1 ? launch(k_paged_short<HD, BITS, 1>, plan.wgs, plan.threads, st, args) : launch(k_paged_short<HD, BITS, SHORT_MORE(HD)>, plan.wgs, plan.threads, st, args);
  const hipError_t e = plan.ct ? launch(k_paged_both<HD, BITS>, plan.wgs, 512, st, args) : launch(k_paged_prompt<HD, BITS>, plan.wgs, 512, st, args);
  return e == hipSuccess && plan.n_splits > 1 ? launch(k_paged_merge<HD>, plan.wgs, 512, st, args, plan.wgs) : e;
}

extern "C" int blink_paged_attention(int32_t device, const blink_paged_attention_args* a, void* stream) {
  g_err.clear();
  if (!a) return fail(BLINK_ERR_INVAL, "null argument");
  if (int rc = check_heads(a->cache, a->n_q_heads)) return rc;
  if (int rc = paged_check(a->cache, a->n_q_heads, a->n_seqs, a->max_q)) return rc;
  const u32 hd = a->cache.head_dim, nkv = a->cache.n_kv_heads;
  const float scale2 = a->scale * 1.44269504088896340736f;      // (scores as powers of two)
  if (!(a->scale > 0.f) || !(scale2 < INFINITY)) return fail(BLINK_ERR_INVAL, "scale must be positive, and finite times log2(e)");
  if (a->sinks && !a->window) return fail(BLINK_ERR_INVAL, "sinks without a window");
  if (a->window > (1u << 30) || a->sinks > (1u << 30)) return fail(BLINK_ERR_INVAL, "window and sinks must be at most 2^30");
  if (a->n_seqs == 0 || a->n_tokens == 0) return BLINK_OK;
  if (!a->max_blocks || a->max_blocks > (1u << 26)) return fail(BLINK_ERR_INVAL, "max_blocks must be in [1, 2^26]");
  if ((u64)a->n_seqs * a->max_blocks * nkv >= (1ull << 31)) return fail(BLINK_ERR_TOO_LARGE, "2^31 blocks of keys or more in one call");
  if ((u64)a->n_tokens * a->n_q_heads >= (1ull << 31)) return fail(BLINK_ERR_TOO_LARGE, "2^31 rows or more");
  if (int rc = check_rows("q", a->q, a->q_stride, (u64)a->n_q_heads * hd, 2)) return rc;
  if (int rc = check_rows("out", a->out, a->out_stride, (u64)a->n_q_heads * hd, 2)) return rc;
  if (!a->cu_seqlens || !a->seq_lens || !a->block_tables) return fail(BLINK_ERR_INVAL, "cu_seqlens, seq_lens and block_tables must not be null");
  if ((u64)a->cu_seqlens % 4 || (u64)a->seq_lens % 4 || (u64)a->block_tables % 4) return fail(BLINK_ERR_INVAL, "cu_seqlens, seq_lens and block_tables must be aligned to 4 bytes");
  u32 n_cu;
  if (int rc = compute_units(device, &n_cu)) return rc;
  const u64 reach = a->window ? (u64)a->window + a->max_q + a->sinks : ~0ull;
  const u32 key_steps = (u32)std::min<u64>(a->max_blocks / 4 + 1, reach / 64 + 3);
  const PagedPlan plan = paged_plan(hd, a->cache.bits, a->n_q_heads, nkv, a->n_seqs, a->n_tokens, a->max_q, key_steps, n_cu);
  if (!a->workspace || (u64)a->workspace % 256 || a->workspace_bytes < plan.bytes(n_cu))
    return fail(BLINK_ERR_INVAL, "a workspace of %llu bytes, aligned to 256, is needed", (unsigned long long)plan.bytes(n_cu));
  OnDevice on(device);
  HIPCHK(on.err);
  PagedArgs p{};
  p.q = (const f16_t*)a->q; p.qs = a->q_stride; p.out = (f16_t*)a->out; p.os = a->out_stride; p.cu = a->cu_seqlens; p.lens = a->seq_lens;
  p.tables = (const u32*)a->block_tables; p.cache = a->cache.data; p.n_blocks = a->cache.n_blocks; p.max_blocks = a->max_blocks;
  p.nq = a->n_q_heads; p.nkv = nkv; p.G = p.nq / nkv; p.n_seqs = a->n_seqs; p.n_tokens = a->n_tokens; p.max_q = a->max_q;
  p.window = a->window; p.sinks = a->sinks; p.c = scale2; p.short_rows = plan.short_rows; p.n_splits = plan.n_splits;
  p.ctr = (u32*)a->workspace; p.part = (float*)((char*)a->workspace + paged_ctr_bytes(n_cu)); p.prompt_part = p.part + plan.part_bytes / 4;
  const hipStream_t st = (hipStream_t)stream;
  HIPCHK(hd == 64 ? (a->cache.bits == 16 ? launch_paged<64, 16>(p, plan, st) : launch_paged<64, 4>(p, plan, st))
                  : (a->cache.bits == 16 ? launch_paged<128, 16>(p, plan, st) : launch_paged<128, 4>(p, plan, st)));
  return BLINK_OK;
}
