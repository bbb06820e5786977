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

extern "C" int blink_kv_cache_copy(int32_t device, const blink_kv_cache* caches, uint32_t n_caches, const int32_t* from_blocks, const int32_t* to_blocks, uint32_t n_copies, void* stream) {
  g_err.clear();
  if (!caches && n_caches) return fail(BLINK_ERR_INVAL, "null argument");
  for (u32 i = 0; i < n_caches; ++i) {
    const blink_kv_cache &c = caches[i], &d = caches[0];
    if (int rc = check_heads(c, c.n_kv_heads)) return rc;
    if (c.n_blocks != d.n_blocks || c.n_kv_heads != d.n_kv_heads || c.head_dim != d.head_dim || c.bits != d.bits) return fail(BLINK_ERR_INVAL, "cache %u is not like the first one", i);
  }
  if (n_copies == 0 || n_caches == 0) return BLINK_OK;
  if (!from_blocks || !to_blocks || (u64)from_blocks % 4 || (u64)to_blocks % 4) return fail(BLINK_ERR_INVAL, "from_blocks or to_blocks is null or not aligned");
  CopyArgs a{};
  a.n_copies = n_copies; a.n_blocks = caches[0].n_blocks; a.from = from_blocks; a.to = to_blocks;
  a.pieces = caches[0].bits == 16 ? 2 : 1;
  a.words = caches[0].n_kv_heads * caches[0].head_dim * (caches[0].bits == 16 ? 32 : 17) / 16;
  a.wgs = (a.words + COPY_WORDS - 1) / COPY_WORDS;
  if ((u64)std::min(n_caches, COPY_CACHES) * n_copies * a.pieces * a.wgs > LAUNCH_WGS) return fail(BLINK_ERR_TOO_LARGE, "too many copies for one call");
  u32 n_cu;
  if (int rc = compute_units(device, &n_cu)) return rc;
  OnDevice on(device);
  HIPCHK(on.err);
  for (u32 done = 0; done < n_caches; done += a.n_caches) {
    a.n_caches = std::min(n_caches - done, COPY_CACHES);
    for (u32 i = 0; i < a.n_caches; ++i) a.cache[i] = caches[done + i].data;
    HIPCHK(launch(k_kv_copy, a.n_caches * n_copies * a.pieces * a.wgs, BLK_THREADS, (hipStream_t)stream, a));
  }
  return BLINK_OK;
}

// ---- log probabilities ----------------------------------------------------------------------------------------------------------
// workgroups of a row: LP_PER_CU for every compute unit in all, a tile for each of their waves at least, and no more keys to join than LP_JOINED
static u32 logprob_parts(u32 rows, u32 vocab, u32 k, u32 n_cu) {
  const u32 tiles = (vocab + LP_WAVES * LP_TILE - 1) / (LP_WAVES * LP_TILE);
  const u64 want = ((u64)LP_PER_CU * n_cu + rows - 1) / rows;
  return rows > LP_CTR_BYTES / 4 ? 1u : (u32)std::min<u64>({want, tiles, LP_MAX_PARTS, LP_JOINED / std::max(k, 1u)});
}
static int check_logprobs(u32 rows, u32 vocab, u32 given, u32 k) {
  if (!vocab || vocab > (1u << 30)) return fail(BLINK_ERR_INVAL, "vocab must be in [1, 2^30]");
  if (given > LP_MOST || k > LP_MOST || k > vocab) return fail(BLINK_ERR_INVAL, "at most %u given tokens, and %u most probable ones of %u", LP_MOST, LP_MOST, vocab);
  if (rows > LAUNCH_WGS) return fail(BLINK_ERR_TOO_LARGE, "too many rows for one call");
  return BLINK_OK;
}
static u64 logprob_bytes(u32 rows, u32 given, u32 k, u32 parts) { return LP_CTR_BYTES + (parts > 1 ? (u64)rows * parts * lp_words(given, k) * 4 : 0); }

extern "C" int blink_token_logprobs_workspace_bytes(int32_t device, uint32_t n_rows, uint32_t vocab, uint32_t n_given, uint32_t k, uint64_t* bytes) {
  g_err.clear();
  if (!bytes) return fail(BLINK_ERR_INVAL, "null argument");
  if (int rc = check_logprobs(n_rows, vocab, n_given, k)) return rc;
  u32 n_cu;
  if (int rc = compute_units(device, &n_cu)) return rc;
  // (and any smaller call's: rows times parts of each are about as many as workgroups are wanted, or fewer)
  const u64 most = std::min<u64>(std::min<u64>(n_rows, LP_CTR_BYTES / 4) * LP_MAX_PARTS, (u64)LP_PER_CU * n_cu + std::min<u64>(n_rows, LP_CTR_BYTES / 4));
  *bytes = LP_CTR_BYTES + most * lp_words(n_given, k) * 4;
  return BLINK_OK;
}

template <typename T>
static hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t st) {
  return a.k ? launch(k_token_logprobs<T, true>, a.rows * a.parts, BLK_THREADS, st, a) : launch(k_token_logprobs<T, false>, a.rows * a.parts, BLK_THREADS, st, a);
}
extern "C" int blink_token_logprobs(int32_t device, const blink_token_logprobs_args* a, void* stream) {
  g_err.clear();
  if (!a) return fail(BLINK_ERR_INVAL, "null argument");
  if (a->type > BLINK_TYPE_BF16) return fail(BLINK_ERR_INVAL, "type must be BLINK_TYPE_FLOAT, BLINK_TYPE_HALF or BLINK_TYPE_BF16");
  if (int rc = check_logprobs(a->n_rows, a->vocab, a->n_given, a->k)) return rc;
  if (a->n_rows == 0) return BLINK_OK;
  if (!a->logits || (u64)a->logits % (a->type == BLINK_TYPE_FLOAT ? 4 : 2)) return fail(BLINK_ERR_INVAL, "logits is null or not aligned to its elements");
  if (a->stride < a->vocab) return fail(BLINK_ERR_INVAL, "a stride of %llu elements, rows are %u long", (unsigned long long)a->stride, a->vocab);
  if (a->n_given && (!a->tokens || !a->logprobs)) return fail(BLINK_ERR_INVAL, "tokens and logprobs must not be null");
  if (a->k && (!a->top_ids || !a->top_logprobs)) return fail(BLINK_ERR_INVAL, "top_ids and top_logprobs must not be null");
  const void* const words[] = {a->tokens, a->inverse_temperature, a->logprobs, a->ranks, a->entropy, a->top_ids, a->top_logprobs};
  for (const void* p : words) if ((u64)p % 4) return fail(BLINK_ERR_INVAL, "tokens, inverse_temperature and the results must be aligned to 4 bytes");
  u32 n_cu;
  if (int rc = compute_units(device, &n_cu)) return rc;
  LogprobArgs l{};
  l.parts = logprob_parts(a->n_rows, a->vocab, a->k, n_cu);
  const u64 need = logprob_bytes(a->n_rows, a->n_given, a->k, l.parts);
  if (!a->workspace || (u64)a->workspace % 256 || a->workspace_bytes < need) return fail(BLINK_ERR_INVAL, "a workspace of %llu bytes, aligned to 256, is needed", (unsigned long long)need);
  OnDevice on(device);
  HIPCHK(on.err);
  l.x = a->logits; l.stride = a->stride; l.rows = a->n_rows; l.V = a->vocab; l.given = a->n_given; l.k = a->k; l.tokens = a->tokens; l.inverse = a->inverse_temperature;
  l.logprobs = a->logprobs; l.ranks = a->n_given ? a->ranks : nullptr; l.entropy = a->entropy; l.top_ids = a->top_ids; l.top_logprobs = a->top_logprobs;
  l.ctr = (u32*)a->workspace; l.results = (u32*)((char*)a->workspace + LP_CTR_BYTES);
  const hipStream_t st = (hipStream_t)stream;
  HIPCHK(a->type == BLINK_TYPE_FLOAT ? launch_logprobs<float>(l, st) : a->type == BLINK_TYPE_HALF ? launch_logprobs<_Float16>(l, st) : launch_logprobs<__bf16>(l, st));
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
static PagedPlan paged_plan(u32 hd, u32 bits, u32 nq, u32 nkv, u32 n_seqs, u32 n_tokens, u32 max_q, u32 steps, u32 n_cu) {
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
  p.n_splits = p.prompt && few ? std::max(1u, steps / 4) : 1u;
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

static void fill_paged(PagedArgs& p, const blink_paged_attention_args* a, float scale2, u32 short_rows, u32 n_splits, u32 n_cu) {
  p.q = (const f16_t*)a->q; p.qs = a->q_stride; p.out = (f16_t*)a->out; p.os = a->out_stride; p.cu = a->cu_seqlens; p.lens = a->seq_lens;
  p.tables = (const u32*)a->block_tables; p.cache = a->cache.data; p.n_blocks = a->cache.n_blocks; p.max_blocks = a->max_blocks;
  p.nq = a->n_q_heads; p.nkv = a->cache.n_kv_heads; p.G = p.nq / p.nkv; p.n_seqs = a->n_seqs; p.n_tokens = a->n_tokens; p.max_q = a->max_q;
  p.window = a->window; p.sinks = a->sinks; p.c = scale2; p.short_rows = short_rows; p.n_splits = n_splits;
  p.ctr = (u32*)a->workspace; p.part = (float*)((char*)a->workspace + paged_ctr_bytes(n_cu));
}
// (nothing: the call has nothing to do)
static int check_attention(const blink_paged_attention_args* a, float* scale2, bool* nothing) {
  if (int rc = check_heads(a->cache, a->n_q_heads)) return rc;
  if (int rc = paged_check(a->cache, a->n_q_heads, a->n_seqs, a->max_q)) return rc;
  const u32 hd = a->cache.head_dim, nkv = a->cache.n_kv_heads;
  *scale2 = a->scale * 1.44269504088896340736f;      // (scores as powers of two)
  if (!(a->scale > 0.f) || !(*scale2 < INFINITY)) return fail(BLINK_ERR_INVAL, "scale must be positive, and finite times log2(e)");
  if (a->sinks && !a->window) return fail(BLINK_ERR_INVAL, "sinks without a window");
  if (a->window > (1u << 30) || a->sinks > (1u << 30)) return fail(BLINK_ERR_INVAL, "window and sinks must be at most 2^30");
  *nothing = a->n_seqs == 0 || a->n_tokens == 0;
  if (*nothing) return BLINK_OK;
  if (!a->max_blocks || a->max_blocks > (1u << 26)) return fail(BLINK_ERR_INVAL, "max_blocks must be in [1, 2^26]");
  if ((u64)a->n_seqs * a->max_blocks * nkv >= (1ull << 31)) return fail(BLINK_ERR_TOO_LARGE, "2^31 blocks of keys or more in one call");
  if ((u64)a->n_tokens * a->n_q_heads >= (1ull << 31)) return fail(BLINK_ERR_TOO_LARGE, "2^31 rows or more");
  if (int rc = check_rows("q", a->q, a->q_stride, (u64)a->n_q_heads * hd, 2)) return rc;
  if (int rc = check_rows("out", a->out, a->out_stride, (u64)a->n_q_heads * hd, 2)) return rc;
  if (!a->cu_seqlens || !a->seq_lens || !a->block_tables) return fail(BLINK_ERR_INVAL, "cu_seqlens, seq_lens and block_tables must not be null");
  if ((u64)a->cu_seqlens % 4 || (u64)a->seq_lens % 4 || (u64)a->block_tables % 4) return fail(BLINK_ERR_INVAL, "cu_seqlens, seq_lens and block_tables must be aligned to 4 bytes");
  return BLINK_OK;
}

// steps of 64 keys of a prompt item, at most
static u32 key_steps(const blink_paged_attention_args* a) {
  const u64 reach = a->window ? (u64)a->window + a->max_q + a->sinks : ~0ull;
  return (u32)std::min<u64>(a->max_blocks / 4 + 1, reach / 64 + 3);
}

extern "C" int blink_paged_attention(int32_t device, const blink_paged_attention_args* a, void* stream) {
  g_err.clear();
  if (!a) return fail(BLINK_ERR_INVAL, "null argument");
  float scale2;
  bool nothing;
  if (int rc = check_attention(a, &scale2, &nothing)) return rc;
  if (nothing) return BLINK_OK;
  const u32 hd = a->cache.head_dim, nkv = a->cache.n_kv_heads;
  u32 n_cu;
  if (int rc = compute_units(device, &n_cu)) return rc;
  const PagedPlan plan = paged_plan(hd, a->cache.bits, a->n_q_heads, nkv, a->n_seqs, a->n_tokens, a->max_q, key_steps(a), n_cu);
  if (!a->workspace || (u64)a->workspace % 256 || a->workspace_bytes < plan.bytes(n_cu))
    return fail(BLINK_ERR_INVAL, "a workspace of %llu bytes, aligned to 256, is needed", (unsigned long long)plan.bytes(n_cu));
  OnDevice on(device);
  HIPCHK(on.err);
  PagedArgs p{};
  fill_paged(p, a, scale2, plan.short_rows, plan.n_splits, n_cu);
  p.prompt_part = p.part + plan.part_bytes / 4;
  const hipStream_t st = (hipStream_t)stream;
  HIPCHK(hd == 64 ? (a->cache.bits == 16 ? launch_paged<64, 16>(p, plan, st) : launch_paged<64, 4>(p, plan, st))
                  : (a->cache.bits == 16 ? launch_paged<128, 16>(p, plan, st) : launch_paged<128, 4>(p, plan, st)));
  return BLINK_OK;
}

// ---- attention of groups --------------------------------------------------------------------------------------------------------
struct SharedPlan {
  u64 part_bytes, prompt_bytes, flat_bytes, row_bytes, token_bytes;
  u64 bytes(u32 n_cu) const { return paged_ctr_bytes(n_cu) + part_bytes + prompt_bytes + flat_bytes + row_bytes + token_bytes; }
};
static SharedPlan shared_plan(u32 hd, const SharedArgs& a, u32 n_cu) {
  SharedPlan p{};
  p.part_bytes = short_floats(n_cu, hd, SHORT_MORE(hd)) * 4;
  p.prompt_bytes = (u64)n_cu * PROMPT_SLOT(hd) * 4;
  p.flat_bytes = 2 * p.prompt_bytes;
  p.row_bytes = 2ull * a.n_rows * a.nq * ROW_RESULT(hd) * 4;
  p.token_bytes = (a.n_tokens + 1ull) * sizeof(JoinToken);
  return p;
}
// waves of the join: one per token and as many query heads as it has lanes for
static u64 join_waves(u32 hd, u32 nq, u32 n_tokens) {
  const u32 heads = hd == 64 ? join_heads<64>() : join_heads<128>();
  return (u64)n_tokens * ((nq + heads - 1) / heads);
}
static int check_groups(const blink_kv_cache& c, u32 nq, u32 n_seqs, u32 n_groups, u32 n_tokens) {
  if ((u64)n_seqs + n_groups > PAGED_MAX_SEQS) return fail(BLINK_ERR_TOO_LARGE, "%u sequences and %u groups, at most %u together in one call", n_seqs, n_groups, PAGED_MAX_SEQS);
  if (n_groups && join_waves(c.head_dim, nq, n_tokens) * 64 + BLK_THREADS > (1ull << 32)) return fail(BLINK_ERR_TOO_LARGE, "%u tokens of %u heads are too many for one call with groups", n_tokens, nq);
  return BLINK_OK;
}

extern "C" int blink_shared_attention_workspace_bytes(int32_t device, const blink_kv_cache* c, uint32_t n_q_heads, uint32_t n_seqs, uint32_t n_groups, uint32_t n_tokens, uint32_t max_q, uint64_t* bytes) {
  if (int rc = blink_attention_workspace_bytes(device, c, n_q_heads, n_seqs, max_q, bytes)) return rc;      // (a call without groups)
  if ((u64)n_tokens * n_q_heads >= (1ull << 31)) return fail(BLINK_ERR_TOO_LARGE, "2^31 rows or more");
  if (int rc = check_groups(*c, n_q_heads, n_seqs, n_groups, n_tokens)) return rc;
  u32 n_cu;
  if (int rc = compute_units(device, &n_cu)) return rc;
  SharedArgs p{};
  p.nq = n_q_heads; p.G = n_q_heads / c->n_kv_heads; p.n_seqs = n_seqs; p.n_tokens = n_tokens; p.max_q = max_q;
  rows_of_call(p);
  *bytes = std::max<u64>(*bytes, shared_plan(c->head_dim, p, n_cu).bytes(n_cu));
  return BLINK_OK;
}

template <int HD, int BITS>
static hipError_t launch_shared(const SharedArgs& args, u32 n_cu, hipStream_t st) {
  constexpr u32 NT = 64 * PAGED_WAVES;
  hipError_t e;
  if constexpr (rows_by_mean(HD, BITS)) e = launch(k_shared_attention<HD, BITS, ANY_CT>, n_cu, NT, st, args);
  else e = args.short_rows == 16 ? launch(k_shared_attention<HD, BITS, 1>, n_cu, NT, st, args) : launch(k_shared_attention<HD, BITS, SHORT_MORE(HD)>, n_cu, NT, st, args);
  const u64 waves = join_waves(HD, args.nq, args.n_tokens);
  return e == hipSuccess ? launch(k_shared_join<HD>, (u32)((waves * 64 + BLK_THREADS - 1) / BLK_THREADS), BLK_THREADS, st, args) : e;
}

extern "C" int blink_shared_attention(int32_t device, const blink_shared_attention_args* s, void* stream) {
  g_err.clear();
  if (!s) return fail(BLINK_ERR_INVAL, "null argument");
  const blink_paged_attention_args* const a = &s->attention;
  float scale2;
  bool nothing;
  if (int rc = check_attention(a, &scale2, &nothing)) return rc;
  if (int rc = check_groups(a->cache, a->n_q_heads, a->n_seqs, s->n_groups, a->n_tokens)) return rc;
  if (nothing) return BLINK_OK;
  if (s->n_groups == 0) return blink_paged_attention(device, a, stream);
  const u32 hd = a->cache.head_dim, nkv = a->cache.n_kv_heads;
  if (((u64)a->n_seqs + s->n_groups) * a->max_blocks * nkv >= (1ull << 31)) return fail(BLINK_ERR_TOO_LARGE, "2^31 blocks of keys or more in one call");
  if (s->share_all > 1) return fail(BLINK_ERR_INVAL, "share_all must be 0 or 1");
  if (!s->group_starts || !s->shared_lens || (u64)s->group_starts % 4 || (u64)s->shared_lens % 4) return fail(BLINK_ERR_INVAL, "group_starts or shared_lens is null or not aligned");
  u32 n_cu;
  if (int rc = compute_units(device, &n_cu)) return rc;
  SharedArgs p{};
  fill_paged(p, a, scale2, 0, std::max(1u, key_steps(a) / 4), n_cu);      // (parts of 256 keys at least)
  rows_of_call(p);
  const SharedPlan plan = shared_plan(hd, p, n_cu);
  if (!a->workspace || (u64)a->workspace % 256 || a->workspace_bytes < plan.bytes(n_cu))
    return fail(BLINK_ERR_INVAL, "a workspace of %llu bytes, aligned to 256, is needed", (unsigned long long)plan.bytes(n_cu));
  OnDevice on(device);
  HIPCHK(on.err);
  p.own_part = p.part + plan.part_bytes / 4;
  p.prompt_part = p.own_part + plan.prompt_bytes / 4;
  p.rows = p.prompt_part + plan.flat_bytes / 4;
  p.tokens = (JoinToken*)(p.rows + plan.row_bytes / 4);
  shared_costs(p, hd, a->cache.bits, n_cu);
  p.n_groups = s->n_groups; p.share_all = s->share_all; p.starts = s->group_starts; p.shared = s->shared_lens;
  const hipStream_t st = (hipStream_t)stream;
  HIPCHK(hd == 64 ? (a->cache.bits == 16 ? launch_shared<64, 16>(p, n_cu, st) : launch_shared<64, 4>(p, n_cu, st))
                  : (a->cache.bits == 16 ? launch_shared<128, 16>(p, n_cu, st) : launch_shared<128, 4>(p, n_cu, st)));
  return BLINK_OK;
}
